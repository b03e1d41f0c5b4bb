// Attention of many query rows per head of keys (trees, chunks of a prompt) over the paged 8-bit cache, bf16: the cached
// tokens on the tensor cores, then the new tokens and the joining of pieces.
//
// Scores. The keys' bytes are multiplied as they lie: tcgen05 takes e4m3 operands at twice bf16's rate, so the queries are
// split in two e4m3 parts, q = hi + lo, and both products are added up in the same fp32 accumulator: the rate of bf16
// without widening a byte. A row is scaled by the power of two that puts its largest element at 2^7..2^8: 4 bits in hi and
// the other 4 of bf16's 8 in lo, exact down to 2^-9 of the largest element and within 2^-17 of it below.
// Output. Splitting the weights the same way costs the softmax more instructions than everything else it does, so the values
// are widened instead (to f16, exactly), once per tile for all rows, and the weights are rounded to f16, as in attn_rows.cu:
// w = 2^(z - m) in fp32 for their sum, P = w v_scale 2^-sh for the product, with sh such that the largest P is 2^7..2^15:
// 11 bits down to 2^-21 of the largest or less.
//
// One CTA per SM takes 128 query rows against tiles of 128 tokens. Everything that the products accumulate or take per row is in
// TMEM, all of its 512 columns: S twice, O, P and the queries. With the queries there, S needs shared memory for the
// keys alone (both operands from there ran at half the rate), and with S twice its products run a tile ahead of the softmax.
// Warp roles:
//   warp 0       pages: TMA copies of a tile's pages and their scales into rings
//   warp 1       MMA issue: S = Q K^T as soon as the softmax has the S of two tiles before in registers, and O += P V (Q and P
//                from TMEM)
//   warps 2, 3   values from e4m3 to f16; what lies behind the last token becomes 0
//   warps 4..19  softmax: four threads per row, 32 columns of S each, which exchange their maxima through shared memory
// O is rescaled only when a row's largest P would pass 2^15, and m moves only when a score passes it by more than 20 (in log2).
// Bounded by the softmax warps' instructions and the chain from S to the next P: 2600 cycles per 128 rows and 128 tokens of 128
// elements, of which the tensor cores need 1100. Trees of 65 nodes of 16 sequences with 1000 to 16384 cached, 32 heads on 8: 284 us,
// 524 TFLOP/s of what is asked for (their 260 rows per head of keys take three tiles of 128; 64 nodes, two tiles: 210 us). Weights
// whose sum shared the values' exponent took 261 us, but their sum depended on the values' scales. At that time products
// issued by two warps, or values widened by one warp or by four at 80 registers, took 314 us.
#include <cuda.h>
#include <cuda_fp16.h>
#include <math.h>

#include "attn_split.cuh"
#include "tc_ptx.cuh"

namespace tf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLow = -3.402823466e38f;      // maximum of nothing yet: no finite score is below it
constexpr float kTop = 8.0f, kSlack = 7.0f;   // log2 of the largest P after a rescale, and its growth until the next
constexpr float kRoom = 20.0f;                // log2 of the largest w
constexpr float kFar = 65536.0f;              // a move of m beyond it leaves little of what was added to it
constexpr float kLeastShift = -200.0f;        // sh where no value counts yet
constexpr int kTile = 128;                    // tokens of a tile
constexpr int kMaxPagesPerTile = 8;
constexpr uint64_t kWaitLimitNs = 2000000000ull;

// ---- sharing out --------------------------------------------------------------------------------------------------
// As in attn_split.cuh, in tiles of 128 tokens of an item of 128 rows, and kStart tiles more for an item's beginning and end
// (its queries, the filling of the pipeline, its output). An item's first piece goes to the item's own rows of the
// workspace, a later one to its CTA's.
constexpr int kStart = 5;
constexpr int kListed = 1024;                 // prefix sums kept: of every sequence, or of every 2nd to 4th

struct WideSplit {
    int rows, row_tiles;                      // rows of (sequence, head); items of 128 of them
    int step;                                 // sequences per listed prefix sum
    int ctas;
    float* base_o;                            // [b * hkv * rows][hd]: a piece's own output (numerators / sum), 0 where there is none
    float2* base_ml;                          // its m and sum of 2^(z - m)
    float* cta_o;                             // [ctas][128][hd]
    float2* cta_ml;
    unsigned long long wait_ns;
};

__device__ __forceinline__ int wide_tiles(const AttnArgs& a, int s) { return (attn_len(a, s) + kTile - 1) / kTile; }
__device__ __forceinline__ long long wide_units(const AttnArgs& a, const WideSplit& p, int s) {
    const int tiles = wide_tiles(a, s);
    return static_cast<long long>(tiles ? tiles + kStart : 0) * a.c.hkv * p.row_tiles;
}

// Units before every step-th sequence in prefix[0 .. ceil(b / step)], the last being all; by one warp.
__device__ __forceinline__ void wide_list(const AttnArgs& a, const WideSplit& p, long long* prefix) {
    const int lane = threadIdx.x & 31, n = (a.c.b + p.step - 1) / p.step;
    long long run = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        long long v = 0;
        for (int s = (i0 + lane) * p.step; s < min((i0 + lane + 1) * p.step, a.c.b); ++s) v += wide_units(a, p, s);
        long long incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (i0 + lane < n) prefix[i0 + lane] = run + incl - v;
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) prefix[n] = run;
}
__device__ __forceinline__ long long wide_total(const AttnArgs& a, const WideSplit& p, const long long* prefix) {
    return prefix[(a.c.b + p.step - 1) / p.step];
}
__device__ __forceinline__ long long wide_before(const AttnArgs& a, const WideSplit& p, const long long* prefix, int s) {
    long long x = prefix[s / p.step];
    for (int i = s / p.step * p.step; i < s; ++i) x += wide_units(a, p, i);
    return x;
}
__device__ __forceinline__ long long wide_share(const WideSplit& p, long long total) {
    const long long even = (total + p.ctas - 1) / p.ctas;
    return even > 1 ? even : 1;
}

struct WideSegment {
    int s, h, rt, t0, t1, len;                // tiles t0..t1-1 of the item's tokens (none if t0 >= t1)
};
// The segment that begins at unit x; moves x behind it.
__device__ __forceinline__ WideSegment wide_segment(const AttnArgs& a, const WideSplit& p, const long long* prefix, long long* x, long long end) {
    WideSegment g;
    const int at = attn_find(prefix, (a.c.b + p.step - 1) / p.step, *x);
    g.s = at * p.step;
    long long local = *x - prefix[at];
    for (long long u; local >= (u = wide_units(a, p, g.s)); ++g.s) local -= u;
    g.len = attn_len(a, g.s);
    const int tiles = (g.len + kTile - 1) / kTile, item = static_cast<int>(local / (tiles + kStart));
    g.h = item / p.row_tiles;
    g.rt = item - g.h * p.row_tiles;
    const int off = static_cast<int>(local - static_cast<long long>(item) * (tiles + kStart));
    const int take = tiles + kStart - off < end - *x ? tiles + kStart - off : static_cast<int>(end - *x);
    g.t0 = max(off - kStart, 0);
    g.t1 = max(off + take - kStart, 0);
    *x += take;
    return g;
}

// ---- PTX ----------------------------------------------------------------------------------------------------------
// Descriptors of shared-memory operands: the low word holds the address (in 16 bytes; advanced by adding to it) and the distance
// of blocks along n, the high word the distance of groups of eight rows, version 1 and the swizzle.
template <int HD>
struct RowDesc {                              // rows of HD bytes under a swizzle as wide as the row
    __device__ __forceinline__ static uint32_t low(uint32_t addr) { return addr >> 4 | 1u << 16; }
    static constexpr uint32_t high = (8 * HD >> 4) | 1u << 14 | (HD == 128 ? 2u : 4u) << 29;
};
constexpr int kVhBlock = kTile * 128;         // f16 values: blocks of 64 elements of rows (tokens) of 128 bytes, 128-byte swizzle
struct VhDesc {
    __device__ __forceinline__ static uint32_t low(uint32_t addr) { return addr >> 4 | static_cast<uint32_t>(kVhBlock >> 4) << 16; }
    static constexpr uint32_t high = (1024u >> 4) | 1u << 14 | 2u << 29;
};
// D[tmem] (+)= A B^T of e4m3 operands: A from TMEM (four elements per column), B from shared memory.
template <uint32_t HIGH>
__device__ __forceinline__ void mma_e4m3_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %4};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
                 "r"(a), "r"(b), "r"(idesc), "n"(HIGH), "r"(static_cast<uint32_t>(accumulate))
                 : "memory");
}
// D[tmem] (+)= A B of f16 operands: A from TMEM (two elements per column), B from shared memory.
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %4};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
                 "r"(a), "r"(b), "r"(idesc), "n"(VhDesc::high), "r"(static_cast<uint32_t>(accumulate))
                 : "memory");
}
// fp32 D, 128 x n, e4m3 (kind::f8f6f4) or f16 (kind::f16) A and B, both with format 0; b_mn: B's rows run along n in memory
// (values: tokens are its rows).
__host__ __device__ constexpr uint32_t idesc_of(int n, bool b_mn) {
    return (1u << 4) | (b_mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | ((128u >> 4) << 24);
}
// Byte offset of 16-byte piece c of row r in a tile of rows of HD bytes.
template <int HD>
__device__ __forceinline__ uint32_t swizzled(int r, int c) {
    return HD == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ (r >> 1 & 3)) << 4);
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_16cols(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_4cols(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Sums rounded toward zero, which no product before them is fused with: the product keeps its own rounding.
__device__ __forceinline__ unsigned long long f2_add_rz(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Two numbers as e4m3 bytes hi + lo, each pair in 16 bits. Their f16 forms (11 bits) are split: hi is the nearest
// e4m3, lo that of the rest.
__device__ __forceinline__ void split2(float x0, float x1, uint16_t* hi, uint16_t* lo) {
    uint32_t h, back;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(x1), "f"(x0));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(*hi) : "r"(h));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(*hi));
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), *reinterpret_cast<const __half2*>(&back));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(*lo) : "r"(*reinterpret_cast<const uint32_t*>(&r)));
}
__device__ __forceinline__ uint32_t join16(uint16_t lo, uint16_t hi) { return static_cast<uint32_t>(hi) << 16 | lo; }

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// True in one lane of a converged warp. Operands that are worked out outside of what it guards stay in uniform registers, where the
// tensor core instructions want them.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

struct PageScale {
    float ks, lv, out, unused;                // keys' scale, log2 of the values'; -inf for a page that is left out, 0 for others
};

template <int HD>
struct WideCfg {
    static constexpr int KST = 4, VST = 3, VHST = 2, SST = 8;   // stages: keys, values as bytes and as f16, scales
    static constexpr int kThreads = 128 + 512;
    static constexpr int kKvBytes = kTile * HD, kVhBytes = 2 * kKvBytes;
    static constexpr int kS = 0, kO = 256, kP = 384, kQ = 448;     // TMEM columns
    static constexpr int kVh = KST * kKvBytes;
    static constexpr int kV = kVh + VHST * kVhBytes;
    static constexpr int kScales = kV + VST * kKvBytes;
    static constexpr int kBars = kScales + SST * kMaxPagesPerTile * sizeof(PageScale);
    static constexpr int kMax = kBars + 512;                       // [2][128][4] pairs: maxima (sums) of a row's four threads
    static constexpr int kPrefix = kMax + 2 * 128 * 32;
    static constexpr size_t smem = kPrefix + (kListed + 1) * 8 + 1024;   // 1024: alignment
};
static_assert(WideCfg<128>::smem <= 227 * 1024, "shared memory");

struct CacheMaps {
    CUtensorMap k, v;
};

template <int HD>
__global__ void __launch_bounds__(WideCfg<HD>::kThreads, 1) wide_attention_kernel(AttnArgs a, WideSplit p, const __grid_constant__ CacheMaps maps) {
    using C = WideCfg<HD>;
    constexpr int KST = C::KST, VST = C::VST, VHST = C::VHST, SST = C::SST;
    extern __shared__ uint8_t raw_smem[];
    uint8_t* smem = raw_smem + ((1024 - (ptx::smem_u32(raw_smem) & 1023)) & 1023);
    PageScale* scales = reinterpret_cast<PageScale*>(smem + C::kScales);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBars);
    uint64_t *k_full = bars, *k_free = k_full + KST, *v_full = k_free + KST, *v_free = v_full + VST, *vh_full = v_free + VST,
             *vh_free = vh_full + VHST, *sc_full = vh_free + VHST, *s_full = sc_full + SST, *s_read = s_full + 2, *p_full = s_read + 2, *p_free = p_full + 1,
             *meet4 = p_free + 1, *q_full = meet4 + 4, *drain = q_full + 1;
    int* abort_flag = reinterpret_cast<int*>(drain + 1);
    uint32_t* tmem_base = reinterpret_cast<uint32_t*>(abort_flag + 1);
    long long* prefix = reinterpret_cast<long long*>(smem + C::kPrefix);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort = abort_flag;
    const uint64_t limit = p.wait_ns ? p.wait_ns : kWaitLimitNs;

    if (threadIdx.x == 0) {
        for (int i = 0; i < KST; ++i) ptx::mbar_init(k_full + i, 1), ptx::mbar_init(k_free + i, 1);
        for (int i = 0; i < VST; ++i) ptx::mbar_init(v_full + i, 1), ptx::mbar_init(v_free + i, 64);
        for (int i = 0; i < VHST; ++i) ptx::mbar_init(vh_full + i, 64), ptx::mbar_init(vh_free + i, 1);
        for (int i = 0; i < SST; ++i) ptx::mbar_init(sc_full + i, 1);
        for (int i = 0; i < 2; ++i) ptx::mbar_init(s_full + i, 1), ptx::mbar_init(s_read + i, 512);
        for (int i = 0; i < 4; ++i) ptx::mbar_init(meet4 + i, 128);
        ptx::mbar_init(p_full, 512);
        ptx::mbar_init(p_free, 1);
        ptx::mbar_init(q_full, 512);
        ptx::mbar_init(drain, 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc(tmem_base, 512);
        ptx::tmem_relinquish();
    }
    if (warp == 2 && lane == 0) ptx::prefetch_tmap(&maps.k), ptx::prefetch_tmap(&maps.v);
    pdl_wait();
    pdl_trigger();                                        // the joining kernel does the new tokens meanwhile
    if (warp == 3) wide_list(a, p, prefix);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_base;
    const long long total = wide_total(a, p, prefix), share = wide_share(p, total);
    const long long x0 = share * blockIdx.x, end = x0 + share < total ? x0 + share : total;
    auto give_up = [&]() {
        *abort = 1;
        set_status(a.status, TF_DEV_TIMEOUT);
    };
    auto wait = [&](uint64_t* bar, uint32_t turn) -> bool {   // the turn-th phase of a barrier, by a whole warp
        return __all_sync(0xffffffffu, ptx::mbar_wait(bar, turn & 1, abort, limit));
    };

    uint32_t k_loaded = 0, v_loaded = 0;                  // (warp 0) tiles whose copies were issued
    if (warp == 0) {
        // ---- pages ------------------------------------------------------------------------------------------------
        const int per_tile = kTile >> a.c.page_log2, nowhere = a.c.n_pages * a.c.hkv * a.c.page;   // no such row: zeros
        const uint64_t pol = ptx::policy_evict_first();
        uint32_t it = 0;
        bool ok = true;
        for (long long x = x0; x < end && ok;) {
            const WideSegment g = wide_segment(a, p, prefix, &x, end);
            if (g.t0 >= g.t1) continue;
            const int32_t* table = a.table + static_cast<size_t>(g.s) * a.c.max_pages;
            const int n_pages = (g.len + a.c.page - 1) >> a.c.page_log2;
            // lane i: page i of a tile. Ids are read two tiles ahead, scales one.
            auto page_of = [&](int t) -> int {
                const int j = t * per_tile + lane;
                int pid = -2;                             // beyond the sequence
                if (lane < per_tile && j < n_pages && t < g.t1) {
                    pid = table[j];
                    if (pid < 0 || pid >= a.c.n_pages) {
                        set_status(a.status + g.s, TF_DEV_BAD_PAGE);
                        pid = -1;
                    }
                }
                return pid;
            };
            float ks = 0.0f, vs = 0.0f;
            auto scales_of = [&](int pid) {
                ks = 0.0f, vs = 0.0f;
                if (pid >= 0) {
                    const size_t chunk = static_cast<size_t>(pid) * a.c.hkv + g.h;
                    ks = a.k_scale[chunk], vs = a.v_scale[chunk];
                }
            };
            int pid = page_of(g.t0), pid_next = page_of(g.t0 + 1);
            scales_of(pid);
            for (int t = g.t0; t < g.t1; ++t, ++it) {
                const float my_ks = ks, my_vs = vs;
                const int my_pid = pid;
                pid = pid_next;
                scales_of(pid);
                pid_next = page_of(t + 2);
                const int kst = it % KST, vst = it % VST, sst = it % SST;
                if (it >= KST) ok = wait(k_free + kst, it / KST - 1);
                if (!ok) break;
                if (lane < per_tile) {
                    // the keys' buffer is free: the scores of KST tiles ago are done, the softmax has read those of two before
                    // that, and with them it had done with the scales of SST tiles ago
                    PageScale sc;
                    sc.ks = my_ks, sc.lv = my_pid >= 0 ? log2f(my_vs) : -INFINITY, sc.out = my_pid >= 0 ? 0.0f : -INFINITY, sc.unused = 0.0f;
                    scales[sst * kMaxPagesPerTile + lane] = sc;
                }
                const int pages = __popc(__ballot_sync(0xffffffffu, my_pid >= -1));   // pages of this tile, from the first on
                const int row = my_pid >= 0 ? (my_pid * a.c.hkv + g.h) << a.c.page_log2 : nowhere;
                const uint32_t bytes = static_cast<uint32_t>(pages) * a.c.page * HD;
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(sc_full + sst), ptx::mbar_arrive_expect_tx(k_full + kst, bytes);
                __syncwarp();
                if (lane < pages)
                    ptx::tma_load_2d(smem + kst * C::kKvBytes + lane * a.c.page * HD, &maps.k, k_full + kst, 0, row, pol);
                k_loaded = it + 1;
                if (it >= VST) ok = wait(v_free + vst, it / VST - 1);
                if (!ok) break;
                if (lane == 0) ptx::mbar_arrive_expect_tx(v_full + vst, bytes);
                __syncwarp();
                if (lane < pages)
                    ptx::tma_load_2d(smem + C::kV + vst * C::kKvBytes + lane * a.c.page * HD, &maps.v, v_full + vst, 0, row, pol);
                v_loaded = it + 1;
            }
        }
        if (!ok) give_up();
    } else if (warp == 1) {
        // ---- products ---------------------------------------------------------------------------------------------
        constexpr uint32_t id_s = idesc_of(kTile, false), id_o = idesc_of(HD, true), high = RowDesc<HD>::high;
        const uint32_t k_low = RowDesc<HD>::low(ptx::smem_u32(smem)), vh_low = VhDesc::low(ptx::smem_u32(smem + C::kVh));
        uint32_t it = 0, n_seg = 0;                       // tiles and segments so far
        bool ok = true;
        auto scores = [&](uint32_t i) -> bool {           // S of the CTA's i-th tile
            const uint32_t kst = i % KST;
            if (!wait(k_full + kst, i / KST)) return false;
            const uint32_t k = k_low + kst * (C::kKvBytes >> 4), d = tmem + C::kS + (i & 1) * 128, q = tmem + C::kQ;
            if (elect_one()) {
#pragma unroll
                for (int j = 0; j < HD / 16; ++j) {       // hi, then lo
                    constexpr int N = HD / 32;
                    mma_e4m3_ts<high>(d, q + 8 * j, k + 2 * (j % N), id_s, j > 0);
                }
                ptx::mma_commit(s_full + (i & 1));
                ptx::mma_commit(k_free + kst);
            }
            __syncwarp();
            return true;
        };
        for (long long x = x0; x < end && ok;) {
            const WideSegment g = wide_segment(a, p, prefix, &x, end);
            if (g.t0 >= g.t1) continue;
            const uint32_t last = it + g.t1 - g.t0;
            ok = wait(q_full, n_seg++);
            if (ok) ptx::tc_fence_after();
            if (ok) ok = scores(it);
            if (ok && it + 1 < last) ok = scores(it + 1);
            for (const uint32_t first = it; it < last && ok; ++it) {
                if (it + 2 < last) ok = wait(s_read + (it & 1), it >> 1);
                if (ok && it + 2 < last) {
                    ptx::tc_fence_after();
                    ok = scores(it + 2);
                }
                const uint32_t vst = it % VHST;
                ok = ok && wait(vh_full + vst, it / VHST) && wait(p_full, it);
                if (!ok) break;
                ptx::tc_fence_after();
                const uint32_t d = tmem + C::kO, w = tmem + C::kP, v = vh_low + vst * (C::kVhBytes >> 4);
                if (elect_one()) {
                    mma_f16_ts(d, w, v, id_o, it > first);
#pragma unroll
                    for (int c = 1; c < kTile / 16; ++c) mma_f16_ts(d, w + 8 * c, v + (16 * 128 >> 4) * c, id_o, true);
                    ptx::mma_commit(p_free);
                    ptx::mma_commit(vh_free + vst);
                }
                __syncwarp();
            }
        }
        if (!ok) give_up();
        __syncwarp();
    } else if (warp < 4) {
        // ---- values to f16 ----------------------------------------------------------------------------------------
        const int tid = threadIdx.x - 64;
        uint32_t it = 0;
        bool ok = true;
        for (long long x = x0; x < end && ok;) {
            const WideSegment g = wide_segment(a, p, prefix, &x, end);
            for (int t = g.t0; t < g.t1; ++t, ++it) {
                const int vst = it % VST, hst = it % VHST, sst = it % SST;
                ok = wait(v_full + vst, it / VST) && wait(sc_full + sst, it / SST) && (it < VHST || wait(vh_free + hst, it / VHST - 1));
                if (!ok) break;
                const uint8_t* from = smem + C::kV + vst * C::kKvBytes;
                uint8_t* to = smem + C::kVh + hst * C::kVhBytes;
                const PageScale* sc = scales + sst * kMaxPagesPerTile;
                const int valid = min(g.len - t * kTile, kTile);
                constexpr int PIECES = HD / 16, EACH = kTile * PIECES / 64;
                auto widen = [&](int r, int c, const uint4& w) {
                    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
                    uint32_t h[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
                            : "=r"(h[2 * k]), "=r"(h[2 * k + 1])
                            : "r"(ww[k]));
                    }
                    uint8_t* at = to + (c >> 2) * kVhBlock;
                    *reinterpret_cast<uint4*>(at + swizzled<128>(r, 2 * (c & 3))) = make_uint4(h[0], h[1], h[2], h[3]);
                    *reinterpret_cast<uint4*>(at + swizzled<128>(r, 2 * (c & 3) + 1)) = make_uint4(h[4], h[5], h[6], h[7]);
                };
                // a lane keeps its piece of the row and goes down the rows
                const int c = tid % PIECES, r0 = tid / PIECES;
                bool all = valid == kTile;
                for (int k = 0; k < kTile >> a.c.page_log2; ++k) all &= sc[k].lv > -INFINITY;
                if (all) {
#pragma unroll
                    for (int i0 = 0; i0 < EACH; i0 += 8) {
                        uint4 w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint4*>(from + swizzled<HD>(r0 + (i0 + i) * (64 / PIECES), c));
#pragma unroll
                        for (int i = 0; i < 8; ++i) widen(r0 + (i0 + i) * (64 / PIECES), c, w[i]);
                    }
                } else {
                    // places behind the last token, and pages without a scale, may hold anything, NaN too: 0 here
                    for (int i = 0; i < EACH; ++i) {
                        const int r = r0 + i * (64 / PIECES);
                        uint4 w = make_uint4(0, 0, 0, 0);
                        if (r < valid && sc[r >> a.c.page_log2].lv > -INFINITY) w = *reinterpret_cast<const uint4*>(from + swizzled<HD>(r, c));
                        widen(r, c, w);
                    }
                }
                fence_async_shared();
                ptx::mbar_arrive(vh_full + hst);
                ptx::mbar_arrive(v_free + vst);
            }
        }
        if (!ok) give_up();
    } else {
        // ---- softmax ----------------------------------------------------------------------------------------------
        const int part = (warp - 4) >> 2;                 // of the row's columns
        const int rr = (warp & 3) * 32 + lane;            // row of the tile = TMEM lane
        const uint32_t lane_at = tmem + (static_cast<uint32_t>(warp & 3) * 32 << 16);
        const uint32_t s_col = lane_at + C::kS + 32 * part, p_col = lane_at + C::kP + 16 * part, o_col = lane_at + C::kO + part * (HD / 4);
        float2* slots = reinterpret_cast<float2*>(smem + C::kMax) + rr * 4;
        uint64_t* meet = meet4 + (warp & 3);
        uint32_t met = 0;
        // what the row's four threads have in place of v: posted, then taken when something else has been done
        auto post = [&](float2 v) {
            slots[(met & 1) * 128 * 4 + part] = v;
            ptx::mbar_arrive(meet);
        };
        auto take = [&](float4 (&all)[2]) -> bool {
            const bool got = wait(meet, met);
            all[0] = *reinterpret_cast<const float4*>(slots + (met & 1) * 128 * 4);
            all[1] = *reinterpret_cast<const float4*>(slots + (met & 1) * 128 * 4 + 2);
            ++met;
            return got;
        };
        auto exchange = [&](float v, float4* all) -> bool {
            float4 two[2];
            post(make_float2(v, 0.0f));
            const bool got = take(two);
            *all = make_float4(two[0].x, two[0].z, two[1].x, two[1].z);
            return got;
        };
        const float zscale = a.scale * kLog2e;
        uint32_t it = 0;                                  // tiles of the CTA so far
        bool ok = true;
        for (long long x = x0; x < end && ok;) {
            const WideSegment g = wide_segment(a, p, prefix, &x, end);
            if (g.t0 >= g.t1) continue;
            const int row = g.rt * 128 + rr;
            const bool rows_here = row - lane < p.rows;   // of this warp: without any, P and what follows from it mean nothing
            float qmul = 0.0f;
            if (rows_here) {
                // queries, scaled and split: each of a row's threads reads and writes a quarter
                constexpr int PIECES = HD / 64;           // of 16 elements
                const bool there = row < p.rows;
                const int node = there ? row / a.c.group : 0;
                const uint4* q = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (static_cast<size_t>(g.s) * a.n + node) * a.q_stride +
                                                                static_cast<size_t>(g.h * a.c.group + (there ? row - node * a.c.group : 0)) * HD) + part * 2 * PIECES;
                uint4 raw[2 * PIECES];
#pragma unroll
                for (int i = 0; i < 2 * PIECES; ++i) raw[i] = there ? q[i] : make_uint4(0, 0, 0, 0);
                uint32_t amax = 0;
#pragma unroll
                for (int i = 0; i < 2 * PIECES; ++i) {
                    const uint32_t ww[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) amax = max(amax, max(ww[j] << 16 & 0x7fff0000u, ww[j] & 0x7fff0000u));
                }
                float4 all;
                ok = exchange(__uint_as_float(amax), &all);
                if (!ok) break;
                amax = max(max(__float_as_uint(all.x), __float_as_uint(all.y)), max(__float_as_uint(all.z), __float_as_uint(all.w)));
                const int e = static_cast<int>(amax >> 23) - 127;
                const int shift = amax == 0 || amax >= 0x7f800000u ? 0 : max(min(7 - e, 126), -120);
                const float up = __uint_as_float(static_cast<uint32_t>(shift + 127) << 23);
                // e4m3 has no infinities, and would cut the row's large elements beside one: such a row's scores are NaN
                qmul = amax >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : __uint_as_float(static_cast<uint32_t>(127 - shift) << 23) * zscale;
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {        // four columns of hi, four of lo
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t ww[4] = {raw[2 * i + k].x, raw[2 * i + k].y, raw[2 * i + k].z, raw[2 * i + k].w};
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint16_t h0, l0, h1, l1;
                            split2(bf16_lo(ww[2 * j]) * up, bf16_hi(ww[2 * j]) * up, &h0, &l0);
                            split2(bf16_lo(ww[2 * j + 1]) * up, bf16_hi(ww[2 * j + 1]) * up, &h1, &l1);
                            hi[2 * k + j] = join16(h0, h1), lo[2 * k + j] = join16(l0, l1);
                        }
                    }
                    tmem_st_4cols(lane_at + C::kQ + 4 * (part * PIECES + i), hi);
                    tmem_st_4cols(lane_at + C::kQ + HD / 4 + 4 * (part * PIECES + i), lo);
                }
                tmem_wait_st();
                ptx::tc_fence_before();
            }
            ptx::mbar_arrive(q_full);
            float m = 0.0f, room = -INFINITY;             // room: the score from which on m moves (at first any)
            float sh = kLeastShift, l = 0.0f;
            uint32_t r[32];                               // this thread's part of the scores
            int valid = 0;                                // tokens there, from the first on
            // of its two groups of 16 tokens: factor of the scores, log2 of the values' scale, -inf for a page that is left out
            float f[2], lv[2], out[2];
            // S of a tile into registers, and to the row's other threads the largest score that this thread has of it and, relative
            // to m, log2 of the largest product of a weight with a scale of values
            auto load = [&](uint32_t i, int t) -> bool {
                if (!(wait(s_full + (i & 1), i >> 1) && wait(sc_full + i % SST, i / SST))) return false;
                if (!rows_here) {
                    ptx::mbar_arrive(s_read + (i & 1));
                    return true;
                }
                ptx::tc_fence_after();
                ptx::tmem_ld_32cols(s_col + (i & 1) * 128, r);
                ptx::tc_fence_before();
                ptx::mbar_arrive(s_read + (i & 1));
                const PageScale* sc = scales + i % SST * kMaxPagesPerTile;
                valid = g.len - t * kTile - 32 * part;
                if (valid < 32) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (e >= valid) r[e] = 0xff800000u;            // -inf, whatever stood there
                }
                float z2[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t* z = r + 16 * k;
                    float mx = max3(__uint_as_float(z[0]), __uint_as_float(z[1]), __uint_as_float(z[2]));
#pragma unroll
                    for (int e = 3; e < 15; e += 2) mx = max3(mx, __uint_as_float(z[e]), __uint_as_float(z[e + 1]));
                    mx = fmaxf(mx, __uint_as_float(z[15]));
                    const PageScale s = sc[(32 * part + 16 * k) >> a.c.page_log2];
                    const bool none = 16 * k >= valid;                 // beyond the last page there is no scale
                    f[k] = none ? 1.0f : qmul * s.ks, lv[k] = none ? 0.0f : s.lv;
                    z2[k] = __fmul_rn(mx, f[k]) + (none ? 0.0f : s.out);   // (-inf where there is none)
                    out[k] = none ? 0.0f : s.out;
                }
                post(make_float2(fmaxf(z2[0], z2[1]), fmaxf(z2[0] - m + lv[0], z2[1] - m + lv[1])));
                return true;
            };
            ok = load(it, g.t0);
            for (int t = g.t0; t < g.t1 && ok; ++t, ++it) {
                if (rows_here) {
                    float4 all[2];
                    ok = take(all);
                    if (!ok) break;
                    const float top = fmaxf(max3(all[0].x, all[0].z, all[1].x), all[1].z);
                    float p_top = fmaxf(max3(all[0].y, all[0].w, all[1].y), all[1].w);
                    if (__any_sync(0xffffffffu, top > room || p_top > sh + (kTop + kSlack))) {
                        if (top > room) {
                            // the numerators, relative to 2^(m + sh), stay as they are
                            const float m2 = ceilf(top), up = m2 - m;
                            p_top -= up;
                            if (room > -INFINITY) l *= ex2(-up), sh -= up;     // (nothing was added to it before)
                            if (fabsf(up) > kFar) {
                                p_top = -INFINITY;                     // nothing is left of it: the largest of the tile's scales bounds it
                                const int pages = (min(g.len - t * kTile, kTile) + a.c.page - 1) >> a.c.page_log2;
#pragma unroll 1
                                for (int k = 0; k < pages; ++k) p_top = fmaxf(p_top, scales[it % SST * kMaxPagesPerTile + k].lv);
                            }
                            m = m2, room = m + kRoom;
                        }
                        // where P would pass 2^15, what this row has goes down
                        const bool moves = p_top > sh + (kTop + kSlack) || sh < kLeastShift;
                        const float sh2 = moves ? fmaxf(ceilf(p_top) - kTop, kLeastShift) : sh, down = ex2(sh - sh2);
                        sh = sh2;
                        if (t > g.t0) {
                            ok = wait(p_free, it - 1);                 // O belongs to the products of the tile before
                            if (!ok) break;
                            ptx::tc_fence_after();
#pragma unroll
                            for (int c = 0; c < HD / 4; c += 16) {
                                uint32_t v[16];
                                ptx::tmem_ld_16cols(o_col + c, v);
#pragma unroll
                                for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * down);
                                tmem_st_16cols(o_col + c, v);
                            }
                        }
                    }
                    uint32_t w[16];                       // 32 weights
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        // (2^126 at most: a weight that would take more is less than 2^-111)
                        const float b = out[k] - m, up = ex2(fminf(lv[k] - sh, 126.0f));
                        const unsigned long long f2 = f2_pack(f[k], f[k]), b2 = f2_pack(b, b), up2 = f2_pack(up, up);
                        float pr[16];
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const unsigned long long arg = f2_add_rz(f2_mul(f2_pack(__uint_as_float(r[16 * k + i]), __uint_as_float(r[16 * k + i + 1])), f2), b2);
                            pr[i] = ex2(f2_lo(arg)), pr[i + 1] = ex2(f2_hi(arg));
                        }
                        if (valid < 32) {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (16 * k + i >= valid) pr[i] = 0.0f;
                        }
                        unsigned long long sum = f2_pack(pr[0], pr[1]);
#pragma unroll
                        for (int i = 2; i < 16; i += 2) sum = f2_add(sum, f2_pack(pr[i], pr[i + 1]));
                        l += f2_lo(sum) + f2_hi(sum);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const unsigned long long p2 = f2_mul(f2_pack(pr[i], pr[i + 1]), up2);
                            const __half2 h = __floats2half2_rn(f2_lo(p2), f2_hi(p2));
                            w[8 * k + i / 2] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                    }
                    // the next tile's scores while the others of this row catch up; P belongs to the products of the tile
                    // before until they are done
                    if (t + 1 < g.t1) ok = load(it + 1, t + 1);
                    if (ok && it > 0) ok = wait(p_free, it - 1);
                    if (!ok) break;
                    tmem_st_16cols(p_col, w);
                    tmem_wait_st();
                    ptx::tc_fence_before();
                } else {
                    // the barriers alone; not to arrive for this tile before the last one's phase is over
                    if (t + 1 < g.t1) ok = load(it + 1, t + 1);
                    if (ok && it > 0) ok = wait(p_free, it - 1);
                    if (!ok) break;
                }
                ptx::mbar_arrive(p_full);
            }
            if (!ok) break;
            ok = wait(p_free, it - 1);                    // the last tile's products
            if (!ok) break;
            if (!rows_here) continue;
            ptx::tc_fence_after();
            float4 all;
            ok = exchange(l, &all);
            if (!ok) break;
            // this piece's output and sum
            const float sum = (all.x + all.y) + (all.z + all.w);
            const size_t at = g.t0 > 0 ? static_cast<size_t>(blockIdx.x) * 128 + rr : (static_cast<size_t>(g.s) * a.c.hkv + g.h) * p.rows + row;
            float* o = (g.t0 > 0 ? p.cta_o : p.base_o) + at * HD + part * (HD / 4);
            if (row < p.rows && part == 0) (g.t0 > 0 ? p.cta_ml : p.base_ml)[at] = make_float2(sum == 0.0f ? kLow : m, sum);
            const float inv = 1.0f / sum, half = ex2(0.5f * sh);       // 2^sh in two steps: it may pass fp32 where the output does not
#pragma unroll
            for (int c = 0; c < HD / 4; c += 16) {
                uint32_t v[16];
                ptx::tmem_ld_16cols(o_col + c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = sum == 0.0f ? 0u : __float_as_uint(__uint_as_float(v[i]) * inv * half * half);
                if (row < p.rows) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(o + c + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
            ptx::tc_fence_before();
        }
        if (!ok) give_up();
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (*abort) {
        // copies and products in flight end before shared memory and TMEM are given back
        if (warp == 0) {
            for (uint32_t i = k_loaded > KST ? k_loaded - KST : 0; i < k_loaded; ++i) ptx::mbar_wait(k_full + i % KST, i / KST & 1, nullptr, kWaitLimitNs);
            for (uint32_t i = v_loaded > VST ? v_loaded - VST : 0; i < v_loaded; ++i) ptx::mbar_wait(v_full + i % VST, i / VST & 1, nullptr, kWaitLimitNs);
        }
        if (warp == 1) {
            if (elect_one()) ptx::mma_commit(drain);      // the lane that issued the products
            __syncwarp();
            ptx::mbar_wait(drain, 0, nullptr, kWaitLimitNs);
        }
        __syncthreads();
    }
    if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

// ---- new tokens, and the pieces together --------------------------------------------------------------------------
// A warp holds 16 query rows: their attention over the new tokens by m16n8k16 bf16 products (weights in two bf16 parts, 16 bits
// and more: one part lost a third of the output's accuracy where the new tokens are all there is), then the cached tokens' pieces are added in their order, and the output is written. The new tokens' keys and values
// are copied to shared memory in chunks of up to 128 (a tree of the usual size is one) and the mask turned into bits, so
// that one wait for memory covers them all. Bounded by latency.
// Many items: a CTA's four warps take 16 rows each. Few (SPREAD): all four take the same 16 rows, each every fourth 16 of the new tokens,
// and then four rows each of the pieces, which are then one wait for memory instead of five: 65 nodes of one sequence over 2000
// cached tokens take 24.6 us with it and 29.0 without, 9 nodes 18.9 and 25.7.
// A prompt of 1024 tokens of one sequence, all of whose work is here, takes 176 us, 49 TFLOP/s: chunks are filled without anything
// in flight for the next one.
constexpr int kJoinWarps = 4;

__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Infinities and NaN of a pair as 0; true if there were any.
__device__ __forceinline__ bool clear_odd(uint32_t& w) {
    const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
    if (lo) w &= 0xffff0000u;
    if (hi) w &= 0x0000ffffu;
    return lo || hi;
}

constexpr int kNewChunk = 128;
__host__ __device__ constexpr int join_row(int hd) { return 2 * hd + 16; }   // bytes of a token in shared memory: rows 16 bytes off
__host__ __device__ inline int join_tokens(int n) { return (min(n, kNewChunk) + 15) / 16 * 16; }
// the new tokens' keys and values; later the rows' numerators in fp32 and 16 factors for each
__host__ __device__ inline size_t join_tile(int n, int hd) {
    const size_t kv = static_cast<size_t>(join_tokens(n)) * 2 * join_row(hd), rows = static_cast<size_t>(16) * kJoinWarps * (hd * 4 + 64);
    return kv > rows ? kv : rows;
}
inline size_t join_smem(int n, int hd) { return join_tile(n, hd) + 16 * kJoinWarps * (kNewChunk / 32) * 4 + (kListed + 1) * 8; }

template <int HD, bool SPREAD>
__global__ void __launch_bounds__(32 * kJoinWarps, 3) join_kernel(AttnArgs a, WideSplit p) {
    extern __shared__ __align__(16) uint8_t join_mem[];
    constexpr int EL = HD / 8, KC = HD / 32, ROW = join_row(HD), ROWS = SPREAD ? 16 : 16 * kJoinWarps;   // rows of the CTA
    const int chunk_tokens = join_tokens(a.n);
    uint8_t* sk = join_mem;
    uint8_t* sv = sk + chunk_tokens * ROW;
    uint32_t* bits = reinterpret_cast<uint32_t*>(join_mem + join_tile(a.n, HD));   // [64 nodes][4]: mask bits of the chunk
    long long* prefix = reinterpret_cast<long long*>(bits + 16 * kJoinWarps * (kNewChunk / 32));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int blocks = (p.rows + ROWS - 1) / ROWS;
    const int sh = blockIdx.x / blocks, s = sh / a.c.hkv, h = sh - s * a.c.hkv;
    const int block0 = (blockIdx.x - sh * blocks) * ROWS, row0 = block0 + (SPREAD ? 0 : 16 * warp);
    const __nv_bfloat16* kp = static_cast<const __nv_bfloat16*>(a.k) + static_cast<size_t>(s) * a.n * a.k_stride + static_cast<size_t>(h) * HD;
    const __nv_bfloat16* vp = static_cast<const __nv_bfloat16*>(a.v) + static_cast<size_t>(s) * a.n * a.v_stride + static_cast<size_t>(h) * HD;
    int row[2], node[2], head[2];
    bool there[2], seen[2] = {false, false};
    uint32_t q[KC][2][4];                                 // [piece of 8 elements][row g, g + 8][word]
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        row[e] = row0 + g + 8 * e;
        there[e] = row[e] < p.rows;
        node[e] = there[e] ? row[e] / a.c.group : 0;
        head[e] = h * a.c.group + (there[e] ? row[e] - node[e] * a.c.group : 0);
        const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (static_cast<size_t>(s) * a.n + node[e]) * a.q_stride +
                                                         static_cast<size_t>(head[e]) * HD);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const uint4 w = there[e] ? qp[t + 4 * c] : make_uint4(0, 0, 0, 0);
            q[c][e][0] = w.x, q[c][e][1] = w.y, q[c][e][2] = w.z, q[c][e][3] = w.w;
        }
    }
    // tokens that any row of the block may see
    const int n_new = a.mask ? a.n : min(block0 + ROWS - 1, p.rows - 1) / a.c.group + 1;
    // tokens j0.. of the chunk (zeros up to a multiple of 16) and its mask bits; all threads call it
    auto fill = [&](int j0) -> bool {
        bool odd = false;
        const int have = min(n_new - j0, kNewChunk), rows = (have + 15) / 16 * 16;
#pragma unroll 4
        for (int i = threadIdx.x; i < rows * (HD / 8); i += 32 * kJoinWarps) {
            const int j = i / (HD / 8), c = i % (HD / 8);
            uint8_t* k_to = sk + j * ROW + 16 * c;
            uint8_t* v_to = sv + j * ROW + 16 * c;
            if (j < have) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(k_to)), "l"(kp + static_cast<size_t>(j0 + j) * a.k_stride + 8 * c) : "memory");
                uint4 v = *reinterpret_cast<const uint4*>(vp + static_cast<size_t>(j0 + j) * a.v_stride + 8 * c);
                odd |= clear_odd(v.x) | clear_odd(v.y) | clear_odd(v.z) | clear_odd(v.w);
                *reinterpret_cast<uint4*>(v_to) = v;
            } else {
                *reinterpret_cast<uint4*>(k_to) = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(v_to) = make_uint4(0, 0, 0, 0);
            }
        }
        // a node's bits, 32 tokens at a time by a whole warp
        const int words = (have + 31) / 32, node0 = block0 / a.c.group, nodes = min(block0 + ROWS - 1, p.rows - 1) / a.c.group - node0 + 1;
#pragma unroll 8
        for (int i = warp; i < nodes * words; i += kJoinWarps) {
            const int nl = i / words, w = i - nl * words, j = j0 + 32 * w + lane;
            const bool see = j < a.n && (a.mask ? a.mask[(static_cast<size_t>(s) * a.n + node0 + nl) * a.n + j] != 0 : j <= node0 + nl);
            const uint32_t b = __ballot_sync(0xffffffffu, see);
            if (lane == 0) bits[nl * (kNewChunk / 32) + w] = b;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return __syncthreads_or(odd);
    };
    // everything before the attention kernel has finished: it lets this one start only after its own wait
    if (warp == 0) wide_list(a, p, prefix);
    bool odd = fill(0);                                   // infinities or NaN among the values
    const long long share = wide_share(p, wide_total(a, p, prefix));
    if (threadIdx.x == 0 && block0 == 0 && h == 0 && attn_len(a, s) != a.seq_len[s]) set_status(a.status + s, TF_DEV_BAD_LENGTH);
    const float zscale = a.scale * kLog2e;
    float o[EL][4], m[2] = {kLow, kLow}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < EL; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    for (int jc = 0; jc < n_new; jc += kNewChunk) {
        if (jc > 0) {
            __syncthreads();                              // the chunk before has been read
            odd = fill(jc);
        }
    const int n_chunk = min(n_new - jc, kNewChunk);
    for (int jl = SPREAD ? 16 * warp : 0; jl < n_chunk; jl += SPREAD ? 16 * kJoinWarps : 16) {
        const int j0 = jc + jl;
        float z[2][4];
        bool see[2][4];                                   // [tokens j0 + 8u + 2t + (i & 1)][row g + 8 (i >> 1)]
        bool any = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t w = there[e] ? bits[(node[e] - block0 / a.c.group) * (kNewChunk / 32) + (jl >> 5)] >> (jl & 16) : 0u;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) see[u][2 * e + i] = w >> (8 * u + 2 * t + i) & 1;
            any |= (w & 0xffffu) != 0;
            seen[e] |= (w & 0xffffu) != 0;
        }
        if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            z[u][0] = z[u][1] = z[u][2] = z[u][3] = 0.0f;
            const uint4* kr = reinterpret_cast<const uint4*>(sk + (jl + 8 * u + g) * ROW);
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const uint4 w = kr[t + 4 * c];
                const uint32_t a0[4] = {q[c][0][0], q[c][1][0], q[c][0][1], q[c][1][1]};
                const uint32_t a1[4] = {q[c][0][2], q[c][1][2], q[c][0][3], q[c][1][3]};
                mma_bf16_16816(z[u], a0, w.x, w.y);
                mma_bf16_16816(z[u], a1, w.z, w.w);
            }
        }
        float top[2] = {kLow, kLow};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[u][i] = see[u][i] ? __fmul_rn(z[u][i], zscale) : -INFINITY;
                top[i >> 1] = fmaxf(top[i >> 1], z[u][i]);
            }
        // bf16 weights may be large: the maximum moves only where it grows by more than 8 (in log2)
        float w[2] = {0.0f, 0.0f};
        bool grows = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
            grows |= top[e] > m[e] + 8.0f;
        }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float m2 = top[e] > m[e] + 8.0f ? top[e] : m[e], f = ex2(m[e] - m2);
                m[e] = m2, l[e] *= f;
#pragma unroll
                for (int i = 0; i < EL; ++i) o[i][2 * e] *= f, o[i][2 * e + 1] *= f;
            }
        }
        uint32_t pa[4], pb[4];                            // the weights, and what bf16 leaves of them
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float pr[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pr[i] = see[u][i] ? ex2(z[u][i] - m[i >> 1]) : 0.0f;
                w[i >> 1] += pr[i];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t h = pack_bf16(pr[2 * e], pr[2 * e + 1]);
                pa[2 * u + e] = h, pb[2 * u + e] = pack_bf16(pr[2 * e] - bf16_lo(h), pr[2 * e + 1] - bf16_hi(h));
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) l[e] += w[e];
        // values: tokens 2t, 2t + 1, 2t + 8, 2t + 9, elements EL g .. EL g + EL - 1
        uint32_t v[4][EL / 2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint4* vr = reinterpret_cast<const uint4*>(sv + (jl + 2 * t + (k & 1) + 8 * (k >> 1)) * ROW + 2 * EL * g);
#pragma unroll
            for (int c = 0; c < EL / 8; ++c) {
                const uint4 x = vr[c];
                v[k][4 * c] = x.x, v[k][4 * c + 1] = x.y, v[k][4 * c + 2] = x.z, v[k][4 * c + 3] = x.w;
            }
        }
#pragma unroll
        for (int i = 0; i < EL; ++i) {
            const uint32_t sel = i & 1 ? 0x7632 : 0x5410;
            const uint32_t b0 = __byte_perm(v[0][i / 2], v[1][i / 2], sel), b1 = __byte_perm(v[2][i / 2], v[3][i / 2], sel);
            mma_bf16_16816(o[i], pa, b0, b1);
            mma_bf16_16816(o[i], pb, b0, b1);
        }
        if (odd) {
            // infinities and NaN reach the rows that see them, and those alone
            for (int k = 0; k < 16 && j0 + k < a.n; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (!there[e] || !attn_sees(a, s, node[e], j0 + k)) continue;
                    const __nv_bfloat16* vr = vp + static_cast<size_t>(j0 + k) * a.v_stride + 2 * EL * t;
#pragma unroll
                    for (int i = 0; i < EL; ++i) {
                        const float v0 = __bfloat162float(vr[i]), v1 = __bfloat162float(vr[EL + i]);
                        if (!isfinite(v0)) o[i][2 * e] += v0;
                        if (!isfinite(v1)) o[i][2 * e + 1] += v1;
                    }
                }
        }
    }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
    }
    // the cached tokens' pieces
    const int tiles = wide_tiles(a, s);
    const int rt = row0 / 128;
    int c0 = 0, c1 = -1;
    if (tiles > 0) {
        const long long first = wide_before(a, p, prefix, s) + (static_cast<long long>(h) * p.row_tiles + rt) * (tiles + kStart) + kStart;
        c0 = static_cast<int>(first / share), c1 = static_cast<int>((first + tiles - 1) / share);
    }
    pdl_wait();
    // The numerators go to shared memory, a row's elements side by side, and the pieces are added as they lie: every load is
    // 512 contiguous bytes. Loops over many rows stay rolled up: this code runs once per CTA, and fetching it is what it waits for first.
    __syncthreads();                                      // keys and values have been read by every warp
    float* rows_o = reinterpret_cast<float*>(join_mem) + warp * 16 * HD;
    float* factors = reinterpret_cast<float*>(join_mem) + kJoinWarps * 16 * HD + warp * 16 * 16;   // [row][piece; 8: of what is there; 9: of the output]
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < EL; i += 4) {
            float* to = rows_o + (g + 8 * e) * HD + 2 * EL * t + i;
            *reinterpret_cast<float4*>(to) = make_float4(o[i][2 * e], o[i + 1][2 * e], o[i + 2][2 * e], o[i + 3][2 * e]);
            *reinterpret_cast<float4*>(to + EL) = make_float4(o[i][2 * e + 1], o[i + 1][2 * e + 1], o[i + 2][2 * e + 1], o[i + 3][2 * e + 1]);
        }
    const bool here = 4 * lane < HD;
    if constexpr (SPREAD) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (t == 0) *reinterpret_cast<float4*>(factors + (g + 8 * e) * 16) = make_float4(m[e], l[e], seen[e] ? 1.0f : 0.0f, 0.0f);
        __syncthreads();
        // four rows of this warp; eight lanes for a row's maxima and sums, all lanes for its numerators
        const float* all_o = reinterpret_cast<const float*>(join_mem);
        const float* all_f = all_o + kJoinWarps * 16 * HD;
        const int at = 4 * warp, mine = at + (lane >> 3), r = row0 + mine, n_rows = min(4, p.rows - row0 - at);
        const bool is = r < p.rows;
        float part[kJoinWarps], top = kLow, sum = 0.0f;
        bool saw = false;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, part[w] = all_f[(16 * w + mine) * 16]);
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) {
            part[w] = ex2(part[w] - top);
            sum = fmaf(all_f[(16 * w + mine) * 16 + 1], part[w], sum);
            saw |= all_f[(16 * w + mine) * 16 + 2] != 0.0f;
        }
        float4 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) {
                const float f = __shfl_sync(0xffffffffu, part[w], 8 * i);
                if (!here) continue;
                const float4 x = *reinterpret_cast<const float4*>(all_o + (16 * w + at + i) * HD + 4 * lane);
                y[i].x = fmaf(x.x, f, y[i].x), y[i].y = fmaf(x.y, f, y[i].y), y[i].z = fmaf(x.z, f, y[i].z), y[i].w = fmaf(x.w, f, y[i].w);
            }
        }
#pragma unroll 1
        for (int cb = c0; cb <= c1; cb += 8) {
            float2 ml = make_float2(kLow, 0.0f);
            const int c_mine = cb + (lane & 7);
            if (c_mine <= c1 && is) ml = c_mine > c0 ? p.cta_ml[static_cast<size_t>(c_mine) * 128 + r - rt * 128] : p.base_ml[static_cast<size_t>(sh) * p.rows + r];
            float4 x[4][8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = cb + k;
                const float* from = (c > c0 ? p.cta_o + (static_cast<size_t>(c) * 128 + row0 + at - rt * 128) * HD
                                            : p.base_o + (static_cast<size_t>(sh) * p.rows + row0 + at) * HD) + 4 * lane;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i][k] = make_float4(0, 0, 0, 0);
                    if (here && c <= c1 && i < n_rows) x[i][k] = *reinterpret_cast<const float4*>(from + i * HD);
                }
            }
            float top2 = ml.x;
#pragma unroll
            for (int o2 = 1; o2 < 8; o2 <<= 1) top2 = fmaxf(top2, __shfl_xor_sync(0xffffffffu, top2, o2));
            top2 = fmaxf(top2, top);
            const float down = ex2(top - top2), f_mine = ml.y * ex2(ml.x - top2);
            float more = f_mine;
#pragma unroll
            for (int o2 = 1; o2 < 8; o2 <<= 1) more += __shfl_xor_sync(0xffffffffu, more, o2);
            top = top2, sum = fmaf(sum, down, more);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = __shfl_sync(0xffffffffu, down, 8 * i);
                y[i].x *= d, y[i].y *= d, y[i].z *= d, y[i].w *= d;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float f = __shfl_sync(0xffffffffu, f_mine, 8 * i + k);
                    y[i].x = fmaf(x[i][k].x, f, y[i].x), y[i].y = fmaf(x[i][k].y, f, y[i].y);
                    y[i].z = fmaf(x[i][k].z, f, y[i].z), y[i].w = fmaf(x[i][k].w, f, y[i].w);
                }
            }
        }
        const bool none = !saw || sum == 0.0f;
        const int nd = is ? r / a.c.group : 0, hq = h * a.c.group + (is ? r - nd * a.c.group : 0);
        if (a.lse && is && (lane & 7) == 0)
            a.lse[(static_cast<size_t>(s) * a.n + nd) * a.c.hq + hq] = none ? -INFINITY : (top + log2f(sum)) * kLn2;
        const float inv_mine = none ? -1.0f : 1.0f / sum;         // negative: the row's output is 0
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float inv = __shfl_sync(0xffffffffu, inv_mine, 8 * i);
            const int node_i = __shfl_sync(0xffffffffu, nd, 8 * i), head_i = __shfl_sync(0xffffffffu, hq, 8 * i);
            if (!here || i >= n_rows) continue;
            uint2 w = make_uint2(0, 0);
            if (!(inv < 0.0f)) w = make_uint2(pack_bf16(y[i].x * inv, y[i].y * inv), pack_bf16(y[i].z * inv, y[i].w * inv));
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + ((static_cast<size_t>(s) * a.n + node_i) * a.c.hq + head_i) * HD + 4 * lane) = w;
        }
        return;
    }
    const int n_rows = min(16, p.rows - row0);
    // eight pieces at a time: their maxima and sums by the row's four lanes, then the numerators
#pragma unroll 1
    for (int cb = c0; cb <= c1; cb += 8) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float2 ml[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int c = cb + t + 4 * k;
                ml[k] = make_float2(kLow, 0.0f);
                if (c <= c1 && there[e])
                    ml[k] = c > c0 ? p.cta_ml[static_cast<size_t>(c) * 128 + row[e] - rt * 128] : p.base_ml[static_cast<size_t>(sh) * p.rows + row[e]];
            }
            float top = fmaxf(ml[0].x, ml[1].x);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)), m[e]);
            const float down = ex2(m[e] - top);
            m[e] = top;
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float f = ml[k].y * ex2(ml[k].x - top);
                factors[(g + 8 * e) * 16 + t + 4 * k] = f;
                sum += f;
            }
            if (t == 0) factors[(g + 8 * e) * 16 + 8] = down;
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            l[e] = l[e] * down + sum;
        }
        __syncwarp();
        const int n = min(8, c1 - cb + 1);
#pragma unroll 1
        for (int r = 0; r < n_rows; r += 4) {
            float4 x[4][8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = cb + k;
                const float* from = (c > c0 ? p.cta_o + (static_cast<size_t>(c) * 128 + row0 + r - rt * 128) * HD
                                            : p.base_o + (static_cast<size_t>(sh) * p.rows + row0 + r) * HD) + 4 * lane;
#pragma unroll
                for (int q2 = 0; q2 < 4; ++q2) {
                    x[q2][k] = make_float4(0, 0, 0, 0);
                    if (here && k < n && r + q2 < n_rows) x[q2][k] = *reinterpret_cast<const float4*>(from + q2 * HD);
                }
            }
#pragma unroll
            for (int q2 = 0; q2 < 4; ++q2) {
                if (!here) continue;
                float4* at = reinterpret_cast<float4*>(rows_o + (r + q2) * HD + 4 * lane);
                const float* f = factors + (r + q2) * 16;
                float4 y = *at;
                y.x *= f[8], y.y *= f[8], y.z *= f[8], y.w *= f[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    y.x = fmaf(x[q2][k].x, f[k], y.x), y.y = fmaf(x[q2][k].y, f[k], y.y), y.z = fmaf(x[q2][k].z, f[k], y.z), y.w = fmaf(x[q2][k].w, f[k], y.w);
                *at = y;
            }
        }
        __syncwarp();
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const bool none = !seen[e] || l[e] == 0.0f;
        if (t == 0) factors[(g + 8 * e) * 16 + 9] = none ? -1.0f : 1.0f / l[e];   // negative: the row's output is 0
        if (a.lse && t == 0 && there[e])
            a.lse[(static_cast<size_t>(s) * a.n + node[e]) * a.c.hq + head[e]] = none ? -INFINITY : (m[e] + log2f(l[e])) * kLn2;
    }
    __syncwarp();
#pragma unroll 1
    for (int r = 0; r < n_rows; ++r) {
        const int nd = (row0 + r) / a.c.group, hq = h * a.c.group + row0 + r - nd * a.c.group;
        const float inv = factors[r * 16 + 9];
        if (!here) continue;
        const float4 y = *reinterpret_cast<const float4*>(rows_o + r * HD + 4 * lane);
        uint2 w = make_uint2(0, 0);
        if (!(inv < 0.0f)) w = make_uint2(pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + ((static_cast<size_t>(s) * a.n + nd) * a.c.hq + hq) * HD + 4 * lane) = w;
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}
// The pool as a matrix of one row per (page, head, token), read one page of one head at a time.
cudaError_t cache_map(CUtensorMap* map, const AttnArgs& a, const void* base) {
    const EncodeTiledFn fn = encode_fn();
    if (!fn) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.c.hd), static_cast<cuuint64_t>(a.c.n_pages) * a.c.hkv * a.c.page};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.c.hd)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(a.c.hd), static_cast<cuuint32_t>(a.c.page)};
    const cuuint32_t es[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          a.c.hd == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

constexpr int kWideCtas = 160;                // at most: one per SM

}  // namespace

// Whether the tensor-core kernel takes these sizes: rows of the pool are counted in 31 bits by its copies.
bool attn_tiles_take(const CacheShape& c) {
    return c.dtype == TF_BF16 && (c.hd == 64 || c.hd == 128) && static_cast<long long>(c.n_pages) * c.hkv * c.page < (1ll << 31) - 256;
}

size_t attn_tiles_ws_bytes(const CacheShape& c, int n) {
    const size_t heads = static_cast<size_t>(c.b) * c.hkv, rows = heads * n * c.group, more = static_cast<size_t>(kWideCtas) * 128;
    return up256(rows * 8) + up256(more * 8) + up256(rows * c.hd * 4) + up256(more * c.hd * 4);
}

cudaError_t launch_attn_tiles(cudaStream_t st, int num_sms, const AttnArgs& a) {
    WideSplit p;
    p.rows = a.n * a.c.group;
    p.row_tiles = (p.rows + 127) / 128;
    p.step = (a.c.b + kListed - 1) / kListed;
    p.ctas = min(num_sms, kWideCtas);
    p.wait_ns = wait_limit_ns();
    const size_t heads = static_cast<size_t>(a.c.b) * a.c.hkv, rows = heads * p.rows, more = static_cast<size_t>(kWideCtas) * 128;
    uint8_t* ws = static_cast<uint8_t*>(a.ws);
    p.base_ml = reinterpret_cast<float2*>(ws);
    p.cta_ml = reinterpret_cast<float2*>(ws += up256(rows * 8));
    p.base_o = reinterpret_cast<float*>(ws += up256(more * 8));
    p.cta_o = reinterpret_cast<float*>(ws += up256(rows * a.c.hd * 4));
    CacheMaps maps;
    cudaError_t e = cache_map(&maps.k, a, a.k_cache);
    if (e == cudaSuccess) e = cache_map(&maps.v, a, a.v_cache);
    if (e != cudaSuccess) return e;
    // few items: all CTAs of 16 rows run at once
    const bool spread = static_cast<long long>(heads) * ((p.rows + 15) / 16) <= 3ll * num_sms;
    auto run = [&](auto kernel, auto join, int threads, size_t smem, std::atomic<uint64_t>& told, std::atomic<uint64_t>& join_told) {
        const cudaError_t r = launch_with_smem(kernel, smem, told, [&] { return launch_pdl(kernel, dim3(p.ctas), dim3(threads), smem, st, a, p, maps); });
        if (r != cudaSuccess) return r;
        const int each = spread ? 16 : 16 * kJoinWarps, blocks = (p.rows + each - 1) / each;
        const dim3 grid(static_cast<unsigned>(heads) * blocks);
        return launch_with_smem(join, join_smem(kNewChunk, a.c.hd), join_told,
                                [&] { return launch_pdl(join, grid, dim3(32 * kJoinWarps), join_smem(a.n, a.c.hd), st, a, p); });
    };
    static std::atomic<uint64_t> done[6];
    if (a.c.hd == 64) {
        if (spread) return run(wide_attention_kernel<64>, join_kernel<64, true>, WideCfg<64>::kThreads, WideCfg<64>::smem, done[0], done[1]);
        return run(wide_attention_kernel<64>, join_kernel<64, false>, WideCfg<64>::kThreads, WideCfg<64>::smem, done[0], done[2]);
    }
    if (spread) return run(wide_attention_kernel<128>, join_kernel<128, true>, WideCfg<128>::kThreads, WideCfg<128>::smem, done[3], done[4]);
    return run(wide_attention_kernel<128>, join_kernel<128, false>, WideCfg<128>::kThreads, WideCfg<128>::smem, done[3], done[5]);
}

}  // namespace tf
