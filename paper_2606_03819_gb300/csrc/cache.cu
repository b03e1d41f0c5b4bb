// The paged 8-bit cache of the verifier's keys and values: lengths, pages and slots (plan) and the writing of new
// tokens with one scale for each page and head (append).
#include <math.h>

#include "verify.cuh"

namespace tf {
namespace {

// ---- plan ---------------------------------------------------------------------------------------------------------
// A handful of integers per sequence and one pool that all sequences share. Which pages a sequence takes or gives
// back follows from two exclusive prefix sums over the sequences (pages given back, pages taken), so one CTA does it
// all: a thread per sequence for the counts and a first page, its warp for more pages than one. Bounded by
// latency: one sequence's growth and its way back (two launches) take 6 us, those of 1000 sequences, an eighth of them prompts of up to
// 2048 tokens with 8 MB of slots, 15 us.
constexpr int kPlanThreads = 1024;
constexpr int kPlanSlots = 2048;         // slots that the same CTA writes; more have a grid of their own. A change and its way back: 1088
                                         // slots 8.1 us (8.5 in a grid), 3400 slots 9.4 (8.6), 17000 slots 14.8 (10.1), 2 M slots 539 (15.5)

struct Change {
    int len, want, have, need, status;   // lengths now and wanted, pages now and wanted
};

__device__ __forceinline__ Change change_of(const CacheShape& c, int len, int delta, int extra, int width) {
    Change x;
    const long long cap = static_cast<long long>(c.max_pages) * c.page;
    long long want = static_cast<long long>(len) + delta + extra;
    if (want < 0) want = 0;
    const bool ok = len >= 0 && len <= cap && want <= cap && want - len <= width;
    x.status = ok ? 0 : TF_DEV_BAD_LENGTH;
    x.len = len;
    x.want = ok ? static_cast<int>(want) : len;
    // a sequence that is refused takes and gives nothing
    x.have = ok ? (len + c.page - 1) >> c.page_log2 : 0;
    x.need = ok ? (x.want + c.page - 1) >> c.page_log2 : 0;
    return x;
}

// Sums over the sequences are of 64 bits: 4096 sequences may ask for 2^27 pages each.
__device__ __forceinline__ long long warp_incl_scan(long long v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// Exclusive prefix of v over the block's threads, and the block's total. All threads call it.
__device__ long long block_excl_scan(long long v, long long* warp_sums, long long* total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
    const long long incl = warp_incl_scan(v);
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const long long w = lane < n_warps ? warp_sums[lane] : 0;
        const long long s = warp_incl_scan(w);
        if (lane < n_warps) warp_sums[lane] = s - w;
        if (lane == 31) warp_sums[32] = s;
    }
    __syncthreads();
    const long long out = warp_sums[warp] + incl - v;
    *total = warp_sums[32];
    __syncthreads();
    return out;
}

// The slots of the new tokens of sequence s, from the table as the plan left it. The old length follows from the new one: a
// sequence whose change was refused (status) kept its length.
__device__ __forceinline__ int added_to(const tf_plan_args& p, int s) {
    const long long grown = static_cast<long long>(p.delta[s]) + p.extra;
    return p.dev_status[s] == 0 && grown > 0 ? static_cast<int>(grown) : 0;
}
__device__ __forceinline__ int slot_of(const CacheShape& c, const tf_plan_args& p, int s, int j, int added, int len) {
    if (j >= added) return -1;
    const int t = len - added + j;
    return p.block_table[static_cast<size_t>(s) * c.max_pages + (t >> c.page_log2)] * c.page + (t & (c.page - 1));
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(CacheShape c, tf_plan_args p, bool slots_too) {
    const int32_t *seq_len = p.seq_len, *delta = p.delta;
    int32_t *table = p.block_table, *free_list = p.free_list;
    const int extra = p.extra, width = p.slot_map ? p.width : 0x7fffffff;
    __shared__ long long warp_sums[33];
    const int tid = threadIdx.x, lane = tid & 31;
    // f(table entry, place in the pool) for the n pages of a lane's sequence s from its j-th on, whose places fall from `at`
    auto each_page = [&](int s, int j, int n, long long at, auto f) {
        if (n > 0) f(table + static_cast<size_t>(s) * c.max_pages + j, at);
        for (uint32_t more = __ballot_sync(0xffffffffu, n > 1); more; more &= more - 1) {
            const int who = __ffs(more) - 1, s2 = __shfl_sync(0xffffffffu, s, who), j2 = __shfl_sync(0xffffffffu, j, who);
            const int n2 = __shfl_sync(0xffffffffu, n, who);
            const long long at2 = __shfl_sync(0xffffffffu, at, who);
            for (int i = 1 + lane; i < n2; i += 32) f(table + static_cast<size_t>(s2) * c.max_pages + j2 + i, at2 - i);
        }
    };
    pdl_wait();
    const int held = min(max(*p.free_count, 0), c.n_pages);

    // pages given back: the i-th of them (in the order of sequences and tokens) goes to place held + R - 1 - i, so
    // that taking as many pages again meets them in the same order
    long long n_back = 0;
    for (int s0 = 0; s0 < c.b; s0 += kPlanThreads) {
        int back = 0;
        long long total;
        if (s0 + tid < c.b) {
            const Change x = change_of(c, seq_len[s0 + tid], delta[s0 + tid], extra, width);
            back = max(x.have - x.need, 0);
        }
        block_excl_scan(back, warp_sums, &total);
        n_back += total;
    }
    if (n_back > 0) {
        long long done = 0;
        for (int s0 = 0; s0 < c.b; s0 += kPlanThreads) {
            int back = 0, need = 0;
            long long total;
            if (s0 + tid < c.b) {
                const Change x = change_of(c, seq_len[s0 + tid], delta[s0 + tid], extra, width);
                back = max(x.have - x.need, 0);
                need = x.need;
            }
            const long long order = block_excl_scan(back, warp_sums, &total);
            each_page(s0 + tid, need, back, held + n_back - 1 - (done + order), [&](int32_t* entry, long long at) {
                if (at < c.n_pages) free_list[at] = *entry;       // more pages than the pool has: nowhere to put them
                *entry = -1;
            });
            done += total;
            __syncthreads();
        }
    }
    const int pool = static_cast<int>(min(held + n_back, static_cast<long long>(c.n_pages)));

    // pages taken: sequence s is served if its pages and those of the sequences before it are there
    long long asked = 0, taken = 0;
    for (int s0 = 0; s0 < c.b; s0 += kPlanThreads) {
        const int s = s0 + tid;
        Change x{0, 0, 0, 0, 0};
        int more = 0;
        long long total;
        if (s < c.b) {
            x = change_of(c, seq_len[s], delta[s], extra, width);
            more = max(x.need - x.have, 0);
        }
        const long long order = asked + block_excl_scan(more, warp_sums, &total);
        const bool served = more == 0 || order + more <= pool;
        const int n_taken = served ? more : 0;
        if (s < c.b) {
            p.new_len[s] = served ? x.want : x.len;
            p.dev_status[s] = x.status | (served ? 0 : TF_DEV_POOL_EMPTY);
        }
        each_page(s, x.have, n_taken, pool - 1 - order, [&](int32_t* entry, long long at) { *entry = free_list[at]; });
        long long total_taken;
        block_excl_scan(n_taken, warp_sums, &total_taken);
        asked += total;
        taken += total_taken;
    }
    if (tid == 0) *p.free_count = static_cast<int>(pool - taken);
    if (slots_too) {
        __syncthreads();                                  // table, lengths and status are the block's own writes
        for (int i = tid; i < c.b * width; i += kPlanThreads) p.slot_map[i] = slot_of(c, p, i / width, i % width, added_to(p, i / width), p.new_len[i / width]);
    }
}

__global__ void slots_kernel(CacheShape c, tf_plan_args p) {
    pdl_wait();
    const int s = blockIdx.y, added = added_to(p, s), len = p.new_len[s];
#pragma unroll 4
    for (int j = blockIdx.x * blockDim.x + threadIdx.x; j < p.width; j += gridDim.x * blockDim.x)
        p.slot_map[static_cast<size_t>(s) * p.width + j] = slot_of(c, p, s, j, added, len);
}

// ---- append -------------------------------------------------------------------------------------------------------
// One CTA per (sequence, page touched, head, keys or values). Each thread holds two groups of 16 elements of the
// page in registers, so the new tokens are read once: their largest magnitude gives the scale, then they are
// converted and written. Bounded by HBM: 3 (bf16) or 5 (fp32) bytes for each element. Four prompts of up to 4173 tokens, 8 heads of
// 128: 99 MB in 21 us (4.8 TB/s), fp32 166 MB in 29 us (5.7 TB/s); 32 accepted paths: 4 us, one launch.
constexpr int kGroup = 16;   // elements of one group: 16 bytes of e4m3

// A group as it was read, so that it takes few registers until it is converted.
template <typename T>
struct Group {
    uint4 v[sizeof(T)];

    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) v[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ float operator[](int e) const {     // (e known at compile time)
        const int word = sizeof(T) == 4 ? e : e / 2;
        const uint4& q = v[word / 4];
        const uint32_t w = word % 4 == 0 ? q.x : word % 4 == 1 ? q.y : word % 4 == 2 ? q.z : q.w;
        return __uint_as_float(sizeof(T) == 4 ? w : e % 2 ? w & 0xffff0000u : w << 16);
    }
};

// Smallest power of two s with amax <= 448 s, at least 2^-100. 448 = 1.75 * 2^8: the exponent of amax goes up by one
// exactly where its mantissa is above 1.75.
__device__ __forceinline__ float scale_for(float amax) {
    if (!(amax > kE4m3Max * kMinScale)) return kMinScale;
    const uint32_t e = (__float_as_uint(amax) + 0x1fffffu) >> 23;   // biased exponent, rounded up above 1.75
    return __uint_as_float((e - 8u) << 23);
}

template <typename T>
__device__ __forceinline__ uint4 to_e4m3(const Group<T>& x, float inv) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = f32_to_e4m3x2(x[4 * i] * inv, x[4 * i + 1] * inv) |
               f32_to_e4m3x2(x[4 * i + 2] * inv, x[4 * i + 3] * inv) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__global__ void append_kernel(CacheShape c, tf_append_args p) {
    const int32_t *slot_map = p.slot_map, *src = p.src;
    const int n_rows = p.n_rows, width = p.width;
    int32_t* status = p.dev_status;
    __shared__ uint32_t warp_max[32];
    const int s = blockIdx.z, t = blockIdx.x, h = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const int tid = threadIdx.x;
    pdl_wait();
    const int32_t* slots = slot_map + static_cast<size_t>(s) * width;
    const int slot0 = slots[0];
    if (slot0 < 0) return;                                  // no new token
    const int lead0 = slot0 & (c.page - 1);
    const int j0 = max(t * c.page - lead0, 0);              // this page's first new token
    if (j0 >= width) return;
    const long long row_stride = is_v ? p.v_stride : p.k_stride;
    const T* rows = static_cast<const T*>(is_v ? p.v : p.k) + static_cast<size_t>(s) * n_rows * row_stride + static_cast<size_t>(h) * c.hd;
    const int per_token = c.hd / kGroup, groups = c.page * per_token;

    Group<T> x[2];
    int at[2], to[2];                                       // this thread's groups: a new one's place, or -1; and its token's slot
    bool row_there[2];
    // the groups of a page that holds `lead` tokens already
    auto fetch = [&](int lead) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int g = tid + i * blockDim.x;
            const int o = g / per_token, part = g - o * per_token, j = j0 + o - lead;
            at[i] = -1;
            if (g >= groups || o < lead || j >= width) continue;
            at[i] = g, to[i] = slots[j];
            const int r = src ? src[static_cast<size_t>(s) * width + j] : j;
            row_there[i] = r >= 0 && r < n_rows;
            if (row_there[i]) x[i].load(rows + static_cast<size_t>(r) * row_stride + part * kGroup);
            else x[i].clear();
        }
    };
    // A sequence's slots run on as a rule, so what its pages hold is known from the first of them, and slots and rows are one wait
    // for memory; other maps are fetched again.
    const int guess = t == 0 ? lead0 : 0;
    fetch(guess);
    const int slot = slots[j0];
    if (slot < 0) return;
    const int pid = slot >> c.page_log2;
    if (pid >= c.n_pages) {
        if (tid == 0) set_status(status + s, TF_DEV_BAD_PAGE);
        return;
    }
    const int lead = slot & (c.page - 1);                   // tokens that the page already holds
    if (lead != guess) fetch(lead);
    const int base = pid * c.page;
    const size_t chunk = (static_cast<size_t>(pid) * c.hkv + h);
    uint8_t* cache = static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + chunk * c.page * c.hd;
    float* scale = (is_v ? p.v_scale : p.k_scale) + chunk;
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (at[i] < 0) continue;
        if (to[i] != base + at[i] / per_token) {            // this page's no longer
            at[i] = -1;
            continue;
        }
        if (!row_there[i]) set_status(status + s, TF_DEV_BAD_PAGE);
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
            const uint32_t a = __float_as_uint(x[i][e]) & 0x7fffffffu;
            if (a < 0x7f800000u) amax = max(amax, a);       // finite values alone decide the scale
        }
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    if ((tid & 31) == 0) warp_max[tid >> 5] = amax;
    const float was = lead > 0 ? *scale : 0.0f;
    __syncthreads();
    amax = 0;
    for (int w = 0; w < static_cast<int>(blockDim.x + 31) / 32; ++w) amax = max(amax, warp_max[w]);
    const float now = fmaxf(was, scale_for(__uint_as_float(amax)));
    const float inv = 1.0f / now;                           // exact: a power of two, or the scale that the caller set
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (at[i] >= 0) reinterpret_cast<uint4*>(cache)[at[i]] = to_e4m3(x[i], inv);
    if (now != was) {
        // tokens of before, at the scale of now
        const float f = was / now;
        for (int g = tid; g < lead * per_token; g += blockDim.x) {
            uint4 w = reinterpret_cast<const uint4*>(cache)[g];
            uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 lo = e4m3x2_to_f32(b[e] & 0xffffu), hi = e4m3x2_to_f32(b[e] >> 16);
                b[e] = f32_to_e4m3x2(lo.x * f, lo.y * f) | f32_to_e4m3x2(hi.x * f, hi.y * f) << 16;
            }
            reinterpret_cast<uint4*>(cache)[g] = make_uint4(b[0], b[1], b[2], b[3]);
        }
        if (tid == 0) *scale = now;                         // read by every thread before the barrier above
    }
}

}  // namespace

cudaError_t launch_cache_plan(cudaStream_t st, const CacheShape& c, const tf_plan_args& p) {
    // few slots are written by the plan's own CTA (one launch instead of two)
    const bool slots_too = p.slot_map && static_cast<long long>(c.b) * p.width <= kPlanSlots;
    const cudaError_t e = launch_pdl(plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, c, p, slots_too);
    if (e != cudaSuccess || !p.slot_map || slots_too) return e;
    const int bx = (p.width + 2047) / 2048;                   // eight slots per thread
    return launch_pdl(slots_kernel, dim3(bx < 64 ? bx : 64, c.b), dim3(256), 0, st, c, p);
}

cudaError_t launch_cache_append(cudaStream_t st, const CacheShape& c, const tf_append_args& p) {
    const int groups = c.page * (c.hd / kGroup);
    const int threads = max(32, ((groups + 1) / 2 + 31) / 32 * 32);   // two groups per thread; 1024 at most (128 x 256)
    const dim3 grid((p.width + c.page - 1) / c.page + 1, 2 * c.hkv, c.b);
    if (c.dtype == TF_BF16) return launch_pdl(append_kernel<__nv_bfloat16>, grid, dim3(threads), 0, st, c, p);
    return launch_pdl(append_kernel<float>, grid, dim3(threads), 0, st, c, p);
}

}  // namespace tf
