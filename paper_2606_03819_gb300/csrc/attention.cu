// Attention of new tokens over a paged 8-bit cache and over themselves: the CUDA-core kernel (fp32, and head sizes
// that the tensor-core kernels do not take) and the kernel that joins split items.
//
// out = sum_t p_t v_t / sum_t p_t with p_t = exp2(z_t - m), z = (scale log2 e) q . k and m the largest z so far: one pass
// over the tokens, in which numerators and sum are rescaled whenever m grows.
#include <math.h>

#include "attn_split.cuh"

namespace tf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---- CUDA-core kernel ---------------------------------------------------------------------------------------------
// A CTA of four warps holds 16 query rows, four per warp. For the scores a lane is a token of a tile of 32, for the
// numerators a lane is every 32nd element of the head. Keys and values are widened to fp32 in shared memory once per
// tile; the keys' rows are padded by four floats, so that the eight lanes of a 16-byte phase meet eight different
// groups of banks. Bounded by shared-memory reads (fp32 has no tensor-core form at full precision), for short contexts by latency: 13
// nodes over 777 tokens of 2 sequences, 16 heads of 64: 22 us with the joining; 4000 tokens: 47 us, 9 TFLOP/s. In bf16 it takes the head
// sizes other than 64 and 128: one token of 64 sequences with up to 32768 cached, size 96, 2.3 ms, 0.7 TB/s.
constexpr int kRows = 16, kTok = 32, kWarps = 4, kRowsPerWarp = kRows / kWarps;   // (a float4 holds a token's weights for a warp)

template <typename T>
__device__ __forceinline__ void widen16(const T* p, float* x);
template <>
__device__ __forceinline__ void widen16<float>(const float* p, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(x)[i] = reinterpret_cast<const float4*>(p)[i];
}
template <>
__device__ __forceinline__ void widen16<__nv_bfloat16>(const __nv_bfloat16* p, float* x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i];
        float4 lo, hi;
        lo.x = __uint_as_float(v.x << 16), lo.y = __uint_as_float(v.x & 0xffff0000u);
        lo.z = __uint_as_float(v.y << 16), lo.w = __uint_as_float(v.y & 0xffff0000u);
        hi.x = __uint_as_float(v.z << 16), hi.y = __uint_as_float(v.z & 0xffff0000u);
        hi.z = __uint_as_float(v.w << 16), hi.w = __uint_as_float(v.w & 0xffff0000u);
        reinterpret_cast<float4*>(x)[2 * i] = lo;
        reinterpret_cast<float4*>(x)[2 * i + 1] = hi;
    }
}
// (u: the piece's place in its row. Eight lanes write eight pieces of a row 64 bytes apart: each begins with another quarter of
// its piece, so that they meet all banks.)
__device__ __forceinline__ void widen16_e4m3(const uint8_t* p, float scale, float* x, int u) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = (i + (u >> 1)) & 3;
        const uint32_t w = at & 2 ? (at & 1 ? v.w : v.z) : (at & 1 ? v.y : v.x);
        const float2 lo = e4m3x2_to_f32(w & 0xffffu), hi = e4m3x2_to_f32(w >> 16);
        reinterpret_cast<float4*>(x)[at] = make_float4(lo.x * scale, lo.y * scale, hi.x * scale, hi.y * scale);
    }
}
__device__ __forceinline__ void zero16(float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(x)[i] = make_float4(0, 0, 0, 0);
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

size_t simt_smem(int b, int hd) {
    return (static_cast<size_t>(kRows) * hd + kTok * (hd + 4) + kTok * hd) * 4 + (static_cast<size_t>(b) + 1) * 8;
}

template <typename T, int ND>   // ND = ceil(hd / 32)
__global__ void __launch_bounds__(32 * kWarps) simt_attention_kernel(AttnArgs a, AttnSplit p) {
    extern __shared__ __align__(16) uint8_t smem[];
    const int hd = a.c.hd, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int kld = hd + 4;
    float* sq = reinterpret_cast<float*>(smem);
    float* sk = sq + kRows * hd;
    float* sv = sk + kTok * kld;
    long long* prefix = reinterpret_cast<long long*>(sv + kTok * hd);
    __shared__ uint8_t bad[kTok];         // tokens of the tile that nothing may see
    __shared__ float4 weights[kWarps][kTok];   // of a warp's four rows

    pdl_wait();
    pdl_trigger();                        // the joining kernel lists the same work meanwhile
    if (warp == 0) attn_list(a, p, prefix);
    __syncthreads();
    const long long total = prefix[a.c.b], share = attn_share(p, total);
    long long x = share * blockIdx.x;
    const long long end = x + share < total ? x + share : total;
    const float zscale = a.scale * kLog2e;
    const int units = hd / 16;

    while (x < end) {
        const Segment g = attn_segment(a, p, prefix, x, end);
        x += g.t1 - g.t0;
        const int len = attn_len(a, g.s);
        if (tid == 0 && len != a.seq_len[g.s]) set_status(a.status + g.s, TF_DEV_BAD_LENGTH);
        const int cached_tiles = (len + kTok - 1) / kTok;
        const int row0 = g.rt * kRows;
        const bool rows_here = row0 + warp * kRowsPerWarp < p.rows;   // of this warp
        __syncthreads();                                    // the item before has been read
        for (int i = tid; i < kRows * units; i += 32 * kWarps) {
            const int r = i / units, u = i - r * units, row = row0 + r;
            float* to = sq + r * hd + 16 * u;
            if (row < p.rows) {
                const int node = row / a.c.group, head = g.h * a.c.group + (row - node * a.c.group);
                widen16<T>(static_cast<const T*>(a.q) + (static_cast<size_t>(g.s) * a.n + node) * a.q_stride +
                               static_cast<size_t>(head) * hd + 16 * u, to);
#pragma unroll
                for (int e = 0; e < 16; ++e) to[e] *= zscale;
            } else {
                zero16(to);
            }
        }
        float m[kRowsPerWarp], l[kRowsPerWarp], o[kRowsPerWarp][ND];
#pragma unroll
        for (int r = 0; r < kRowsPerWarp; ++r) {
            m[r] = -INFINITY, l[r] = 0.0f;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[r][d] = 0.0f;
        }
        for (int t = g.t0; t < g.t1; ++t) {
            const bool cached = t < cached_tiles;
            const int tok0 = cached ? t * kTok : (t - cached_tiles) * kTok;
            if (t > g.t0) __syncthreads();                  // the tile before has been read
            for (int i = tid; i < 2 * kTok * units; i += 32 * kWarps) {
                const int is_v = i >= kTok * units, ii = i - (is_v ? kTok * units : 0);
                const int tt = ii / units, u = ii - tt * units, tok = tok0 + tt;
                float* to = (is_v ? sv + tt * hd : sk + tt * kld) + 16 * u;
                bool good = true;
                if (tok >= (cached ? len : a.n)) {
                    good = false;
                } else if (cached) {
                    const int pid = a.table[static_cast<size_t>(g.s) * a.c.max_pages + (tok >> a.c.page_log2)];
                    if (pid < 0 || pid >= a.c.n_pages) {
                        good = false;
                        set_status(a.status + g.s, TF_DEV_BAD_PAGE);
                    } else {
                        const size_t chunk = static_cast<size_t>(pid) * a.c.hkv + g.h;
                        const size_t at = (chunk * a.c.page + (tok & (a.c.page - 1))) * hd + 16 * u;
                        widen16_e4m3((is_v ? a.v_cache : a.k_cache) + at, (is_v ? a.v_scale : a.k_scale)[chunk], to, u);
                    }
                } else {
                    widen16<T>(static_cast<const T*>(is_v ? a.v : a.k) + (static_cast<size_t>(g.s) * a.n + tok) * (is_v ? a.v_stride : a.k_stride) +
                                   static_cast<size_t>(g.h) * hd + 16 * u, to);
                }
                if (!good) zero16(to);
                if (!is_v && u == 0) bad[tt] = !good;
            }
            __syncthreads();
            if (!rows_here) continue;
            float z[kRowsPerWarp] = {};
            const float* kt = sk + lane * kld;
            const float* qt = sq + warp * kRowsPerWarp * hd;
            for (int d = 0; d < hd; d += 4) {
                const float4 kv = *reinterpret_cast<const float4*>(kt + d);
#pragma unroll
                for (int r = 0; r < kRowsPerWarp; ++r) {
                    const float4 qv = *reinterpret_cast<const float4*>(qt + r * hd + d);
                    z[r] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, z[r]))));
                }
            }
            float pr[kRowsPerWarp];
#pragma unroll
            for (int r = 0; r < kRowsPerWarp; ++r) {
                const int row = row0 + warp * kRowsPerWarp + r;
                bool see = row < p.rows && !bad[lane];
                if (see && !cached) see = attn_sees(a, g.s, row / a.c.group, tok0 + lane);
                const float zz = see ? z[r] : -INFINITY;
                const float m2 = fmaxf(m[r], warp_max(zz));
                const float base = m2 == -INFINITY ? 0.0f : m2;
                const float f = exp2f(m[r] - base);
                pr[r] = see ? exp2f(zz - base) : 0.0f;
                l[r] = l[r] * f + warp_sum(pr[r]);
                m[r] = m2;
#pragma unroll
                for (int d = 0; d < ND; ++d) o[r][d] *= f;
            }
            weights[warp][lane] = make_float4(pr[0], pr[1], pr[2], pr[3]);
            __syncwarp();
#pragma unroll 4
            for (int tt = 0; tt < kTok; ++tt) {
                float v[ND];
#pragma unroll
                for (int d = 0; d < ND; ++d) v[d] = lane + 32 * d < hd ? sv[tt * hd + lane + 32 * d] : 0.0f;
                const float4 w4 = weights[warp][tt];
                const float w[kRowsPerWarp] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int r = 0; r < kRowsPerWarp; ++r)
                    if (w[r] != 0.0f) {                     // an unseen token's value may be NaN
#pragma unroll
                        for (int d = 0; d < ND; ++d) o[r][d] = fmaf(w[r], v[d], o[r][d]);
                    }
            }
            __syncwarp();
        }
        const bool whole = g.t0 == 0 && g.t1 == g.tiles;
        const int slot = attn_slot(blockIdx.x, g.t0);
#pragma unroll
        for (int r = 0; r < kRowsPerWarp; ++r) {
            const int rr = warp * kRowsPerWarp + r, row = row0 + rr;
            if (row >= p.rows) continue;
            const int node = row / a.c.group, head = g.h * a.c.group + (row - node * a.c.group);
            if (!attn_row_present(a, g.s, node)) m[r] = -INFINITY, l[r] = 0.0f;
            const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
            if (whole) {
                const size_t at = (static_cast<size_t>(g.s) * a.n + node) * a.c.hq + head;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    if (lane + 32 * d < hd)
                        static_cast<T*>(a.out)[at * hd + lane + 32 * d] = from_f32<T>(l[r] == 0.0f ? 0.0f : o[r][d] * inv);
                if (a.lse && lane == 0) a.lse[at] = l[r] == 0.0f ? -INFINITY : (m[r] + log2f(l[r])) * kLn2;
            } else {
                const size_t at = static_cast<size_t>(slot) * p.rt + rr;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    if (lane + 32 * d < hd) p.part_o[at * hd + lane + 32 * d] = l[r] == 0.0f ? 0.0f : o[r][d] * inv;
                if (lane == 0) p.part_ml[at] = make_float2(m[r], l[r]);
            }
        }
    }
}

// ---- joining split items ------------------------------------------------------------------------------------------
// Weighs each piece's output of a row by its sum, times exp2 of its maximum against the largest. Few items are cut in many
// pieces: a CTA per row then, its warps sharing the pieces (SPREAD); many items in few: a warp per row.
// The kernel before lets this one start early, so the work is listed while that one runs: everything before it on the
// stream has then finished, and it does not write what is read for that (seq_len).
constexpr int kJoinWarps = 8;
constexpr int kAtOnce = 4;               // pieces whose loads are in flight together

template <typename T, bool SPREAD>
__global__ void __launch_bounds__(32 * kJoinWarps) combine_kernel(AttnArgs a, AttnSplit p) {
    extern __shared__ long long prefix[];
    __shared__ __align__(16) float so[SPREAD ? kJoinWarps : 1][SPREAD ? kMaxHeadDim : 4];
    __shared__ float2 sml[kJoinWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hd = a.c.hd;
    if (warp == 0) attn_list(a, p, prefix);
    __syncthreads();
    const long long share = attn_share(p, prefix[a.c.b]);
    const int per_block = SPREAD ? 1 : kJoinWarps, blocks_per_item = (p.rt + per_block - 1) / per_block;
    const int per_seq = a.c.hkv * p.row_tiles;
    const int item = blockIdx.x / blocks_per_item;
    const int rr = (blockIdx.x - item * blocks_per_item) * per_block + (SPREAD ? 0 : warp);
    const int s = item / per_seq, in_seq = item - s * per_seq;
    const int h = in_seq / p.row_tiles, row = (in_seq - h * p.row_tiles) * p.rt + rr;
    const int tiles = attn_tiles(a, p, s);
    const long long first = prefix[s] + static_cast<long long>(in_seq) * tiles;
    const int c0 = static_cast<int>(first / share), c1 = static_cast<int>((first + tiles - 1) / share);
    pdl_wait();
    if (c0 == c1 || rr >= p.rt || row >= p.rows) return;    // one CTA had all of it, or there is no such row
    // this warp's pieces: first_c, first_c + step, ...
    const int step = SPREAD ? kJoinWarps : 1, first_c = c0 + (SPREAD ? warp : 0);
    float m = -INFINITY;
    for (int c = first_c + step * lane; c <= c1; c += 32 * step)
        m = fmaxf(m, p.part_ml[static_cast<size_t>(2 * c + (c == c0)) * p.rt + rr].x);
    m = warp_max(m);
    float base = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    float4 o[2] = {};                                       // elements 4 lane and 128 + 4 lane of the head
    for (int cb = first_c; cb <= c1; cb += 32 * step) {
        float f = 0.0f;                                     // the weight of this lane's piece
        const int mine = cb + step * lane;
        if (mine <= c1) {
            const float2 ml = p.part_ml[static_cast<size_t>(2 * mine + (mine == c0)) * p.rt + rr];
            f = ml.y == 0.0f ? 0.0f : ml.y * exp2f(ml.x - base);
            l += f;
        }
        const int n = min(32, (c1 - cb) / step + 1);
        for (int j = 0; j < n; j += kAtOnce) {
            float4 v[kAtOnce][2];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int c = cb + (j + k) * step;
                const float* from = p.part_o + (static_cast<size_t>(2 * c + (c == c0)) * p.rt + rr) * hd + 4 * lane;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    v[k][i] = make_float4(0, 0, 0, 0);
                    if (j + k < n && 128 * i + 4 * lane < hd) v[k][i] = *reinterpret_cast<const float4*>(from + 128 * i);
                }
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const float w = __shfl_sync(0xffffffffu, f, (j + k) & 31);
                if (j + k >= n || w == 0.0f) continue;      // a piece in which the row saw nothing
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    o[i].x = fmaf(v[k][i].x, w, o[i].x), o[i].y = fmaf(v[k][i].y, w, o[i].y);
                    o[i].z = fmaf(v[k][i].z, w, o[i].z), o[i].w = fmaf(v[k][i].w, w, o[i].w);
                }
            }
        }
    }
    l = warp_sum(l);
    if constexpr (SPREAD) {
        // the warps' parts, by the first warp
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (128 * i + 4 * lane < hd) *reinterpret_cast<float4*>(&so[warp][128 * i + 4 * lane]) = o[i];
        if (lane == 0) sml[warp] = make_float2(m, l);
        __syncthreads();
        if (warp > 0) return;
        m = warp_max(lane < kJoinWarps ? sml[lane].x : -INFINITY);
        base = m == -INFINITY ? 0.0f : m;
        l = 0.0f;
        o[0] = o[1] = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) {
            const float2 ml = sml[w];
            if (ml.y == 0.0f) continue;
            const float f = exp2f(ml.x - base);
            l = fmaf(ml.y, f, l);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (128 * i + 4 * lane < hd) {
                    const float4 v = *reinterpret_cast<const float4*>(&so[w][128 * i + 4 * lane]);
                    o[i].x = fmaf(v.x, f, o[i].x), o[i].y = fmaf(v.y, f, o[i].y);
                    o[i].z = fmaf(v.z, f, o[i].z), o[i].w = fmaf(v.w, f, o[i].w);
                }
        }
    }
    const int node = row / a.c.group, head = h * a.c.group + (row - node * a.c.group);
    const size_t at = (static_cast<size_t>(s) * a.n + node) * a.c.hq + head;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    T* out = static_cast<T*>(a.out) + at * hd;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (128 * i + 4 * lane < hd) {
            T* to = out + 128 * i + 4 * lane;
            to[0] = from_f32<T>(o[i].x * inv), to[1] = from_f32<T>(o[i].y * inv);
            to[2] = from_f32<T>(o[i].z * inv), to[3] = from_f32<T>(o[i].w * inv);
        }
    if (a.lse && lane == 0) a.lse[at] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <typename T>
cudaError_t launch_simt(cudaStream_t st, const AttnArgs& a, const AttnSplit& p, size_t smem) {
    static std::atomic<uint64_t> done[3];
    auto run = [&](auto kernel, std::atomic<uint64_t>& told) {
        return launch_with_smem(kernel, simt_smem(kMaxCacheBatch, kMaxHeadDim), told,
                                [&] { return launch_pdl(kernel, dim3(p.ctas), dim3(32 * kWarps), smem, st, a, p); });
    };
    if (a.c.hd <= 64) return run(simt_attention_kernel<T, 2>, done[0]);
    if (a.c.hd <= 128) return run(simt_attention_kernel<T, 4>, done[1]);
    return run(simt_attention_kernel<T, 8>, done[2]);
}

// From 17 rows on the tensor cores' tiles of 128 rows: the kernel for few rows takes 16 at once and would read the cache again
// for every 16 more. 20 rows over 16 sequences of up to 16384 tokens: 92 us there, 162 here. (Over one of 2000 tokens the two are
// near each other, 18 and 16 us; lengths are not known on the host.)
bool many_rows(const CacheShape& c, int n) { return static_cast<long long>(n) * c.group > 16 && attn_tiles_take(c); }

}  // namespace

cudaError_t launch_attn_combine(cudaStream_t st, const AttnArgs& a, const AttnSplit& p) {
    const long long items = static_cast<long long>(a.c.b) * a.c.hkv * p.row_tiles;
    const size_t smem = (static_cast<size_t>(a.c.b) + 1) * 8;
    // from 8 pieces per item on average the warps of a CTA share them
    const bool spread = items * 8 <= p.ctas;
    const int per_block = spread ? 1 : kJoinWarps;
    const dim3 grid(static_cast<unsigned>(items * ((p.rt + per_block - 1) / per_block)));
    auto run = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(32 * kJoinWarps), smem, st, a, p); };
    if (a.c.dtype == TF_BF16) return spread ? run(combine_kernel<__nv_bfloat16, true>) : run(combine_kernel<__nv_bfloat16, false>);
    return spread ? run(combine_kernel<float, true>) : run(combine_kernel<float, false>);
}

size_t attention_ws_bytes(const CacheShape& c, int n) {
    if (many_rows(c, n)) return attn_tiles_ws_bytes(c, n);
    return attn_part_bytes(kRows, c.hd);
}

cudaError_t launch_tree_attention(cudaStream_t st, int num_sms, const AttnArgs& a) {
    AttnSplit p;
    p.rows = a.n * a.c.group;
    if (many_rows(a.c, a.n)) return launch_attn_tiles(st, num_sms, a);
    if (a.c.dtype == TF_BF16 && (a.c.hd == 64 || a.c.hd == 128)) return launch_attn_rows(st, num_sms, a, p);
    p.row_tiles = (p.rows + kRows - 1) / kRows;
    p.tile_tokens = kTok;
    p.min_tiles = 1;
    p.ctas = kAttnMaxCtas;
    p.rt = kRows;
    attn_place_parts(a, &p);
    const size_t smem = simt_smem(a.c.b, a.c.hd);
    const cudaError_t e = a.c.dtype == TF_BF16 ? launch_simt<__nv_bfloat16>(st, a, p, smem) : launch_simt<float>(st, a, p, smem);
    if (e != cudaSuccess) return e;
    return launch_attn_combine(st, a, p);
}

}  // namespace tf
