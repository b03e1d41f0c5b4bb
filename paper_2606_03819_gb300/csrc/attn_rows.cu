// Attention of few query rows per head of keys (plain decoding, small trees) over the paged 8-bit cache, bf16.
//
// With at most 16 rows the work is to read the cache once: two bytes per token and element for 4 rows FLOPs. Every warp
// therefore loads its tokens' bytes from global memory straight into the fragments of m16n8k16 products - no shared
// memory and no barrier in the loop - and keeps a running maximum, sum and output of its own; the four warps of a CTA
// are joined at the end of an item. The products are transposed, so that tokens (then head elements) fill the 16 rows
// of a fragment and 8 or 16 query rows its columns:
//   S^T [16 tokens x rows] = K Q^T,   O^T [16 elements x rows] += V^T P^T
// Which element of a head stands at which index of a product is free as long as both operands agree, so a lane takes 16
// consecutive bytes of a token's key (of four tokens' values) and no byte has to change lanes; only P^T is
// transposed between the two products, 8 x 8 at a time.
//
// e4m3 widens to f16 exactly. Queries are bf16 numbers times a power of two per row that puts the row's largest
// element at 2^14..2^15: exact for elements down to 2^-24 of it, those below lose bits that are less than 2^-38
// of the largest. A page's scale of keys multiplies the scores z. The weights are those of the scores alone, in fp32,
//   w = 2^(z - m),  m the largest score so far, rounded up,   sum of weights = sum w,
// so that the values' scales cannot make their sum overflow or vanish. For the product they take the page's scale of values and
// are rounded to f16,
//   P = w v_scale 2^-sh,  sh whole, such that the largest P so far is 2^13..2^14,
// which keeps f16's 11 bits down to 2^-27 of the largest term of the output. m and sh are whole numbers: what is summed so far
// is moved by powers of two, without rounding.
//
// Bounded by HBM: one token of 64 sequences with up to 32768 cached (32 heads on 8, size 128; 2.15 GB) takes 349 us, 6.2 TB/s, with
// two CTAs per SM and 250 registers; three at 168 registers spill and take 597. (With 9 to 16 rows of size 128 even 255 are too few: 104
// bytes are spilled; four tokens of the same sequences take 542 us.) One sequence with 4100 cached: 10.6 us, a chain of page ids,
// scales and bytes, then the joining.
#include <cuda_fp16.h>
#include <math.h>

#include "attn_split.cuh"

namespace tf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWarps = 4;
constexpr int kTok = 32;                  // tokens of one warp per step: two fragments of 16
constexpr int kTile = kTok * kWarps;      // tokens of one CTA per step
constexpr float kLow = -3.402823466e38f;  // maximum of nothing yet: no finite score is below it
constexpr float kHead = 14.0f;            // log2 of the largest P
constexpr float kLeastShift = -200.0f;    // sh where no value counts yet

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t widen2(uint32_t two) {   // two e4m3 bytes (low half) to f16x2
    uint32_t h;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
__device__ __forceinline__ uint32_t widen2_hi(uint32_t two) {
    uint32_t h;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 ldg16(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ldg8(const uint8_t* p) {
    uint2 v;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}

// The bytes of one warp's 32 tokens, and their pages' scales.
template <int HD>
struct Tokens {
    static constexpr int KC = HD / 64;        // 16-byte pieces of a key per lane
    static constexpr int VW = HD / 32;        // words of a value per lane
    uint32_t k[2][2][KC][4];                  // [fragment][token g, g + 8][piece][word]
    uint32_t v[2][4][VW];                     // [fragment][tokens 2t, 2t + 1, 2t + 8, 2t + 9][word]
    float ks[2], vs[2];
    int n[2];                                 // tokens that there are (the first n of 16)

    // page ids of the warp's two fragments (which lie in one page each); -1: none or a bad one
    __device__ __forceinline__ void load(const AttnArgs& a, const int (&pid)[2], int h, int tok, int len) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int left = len - (tok + 16 * f);
            n[f] = pid[f] < 0 || left <= 0 ? 0 : left < 16 ? left : 16;
            const size_t chunk = static_cast<size_t>(pid[f] < 0 ? 0 : pid[f]) * a.c.hkv + h;
            const size_t base = (chunk * a.c.page + ((tok + 16 * f) & (a.c.page - 1))) * HD;
            ks[f] = n[f] ? a.k_scale[chunk] : 0.0f;
            vs[f] = n[f] ? a.v_scale[chunk] : 1.0f;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (g + 8 * e < n[f]) w = ldg16(a.k_cache + base + (g + 8 * e) * HD + 16 * (t + 4 * c));
                    k[f][e][c][0] = w.x, k[f][e][c][1] = w.y, k[f][e][c][2] = w.z, k[f][e][c][3] = w.w;
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int tk = 2 * t + (e & 1) + 8 * (e >> 1);
                const uint8_t* p = a.v_cache + base + tk * HD + 4 * VW * g;
                if constexpr (VW == 4) {
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (tk < n[f]) w = ldg16(p);
                    v[f][e][0] = w.x, v[f][e][1] = w.y, v[f][e][2] = w.z, v[f][e][3] = w.w;
                } else {
                    uint2 w = make_uint2(0, 0);
                    if (tk < n[f]) w = ldg8(p);
                    v[f][e][0] = w.x, v[f][e][1] = w.y;
                }
            }
        }
    }
};

__device__ __forceinline__ void page_ids(const AttnArgs& a, int s, int tok, int len, int (&pid)[2]) {
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        pid[f] = -1;
        if (tok + 16 * f < len) {
            pid[f] = a.table[static_cast<size_t>(s) * a.c.max_pages + ((tok + 16 * f) >> a.c.page_log2)];
            if (pid[f] < 0 || pid[f] >= a.c.n_pages) {
                set_status(a.status + s, TF_DEV_BAD_PAGE);
                pid[f] = -1;
            }
        }
    }
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// NT: blocks of 8 query rows.
template <int HD, int NT>
__global__ void __launch_bounds__(32 * kWarps, 2) rows_attention_kernel(AttnArgs a, AttnSplit p) {
    constexpr int KS = HD / 16;               // products along a key
    constexpr int MT = HD / 16;               // fragments of 16 head elements
    constexpr int R = 8 * NT;
    constexpr int EL = HD / 8;                // head elements of one lane: EL g .. EL g + EL - 1
    extern __shared__ long long prefix[];
    __shared__ __align__(16) float so[kWarps][R][HD];
    __shared__ float2 sml[kWarps][R];
    __shared__ float ssh[kWarps][R];
    __shared__ uint8_t present[R];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;

    pdl_wait();
    pdl_trigger();                            // the joining kernel lists the same work meanwhile
    if (warp == 0) attn_list(a, p, prefix);
    __syncthreads();
    const long long total = prefix[a.c.b], share = attn_share(p, total);
    long long x = share * blockIdx.x;
    const long long end = x + share < total ? x + share : total;
    const float zscale = a.scale * kLog2e;

    while (x < end) {
        const Segment sg = attn_segment(a, p, prefix, x, end);
        x += sg.t1 - sg.t0;
        const int len = attn_len(a, sg.s);
        if (threadIdx.x == 0 && len != a.seq_len[sg.s]) set_status(a.status + sg.s, TF_DEV_BAD_LENGTH);
        const int cached_tiles = (len + kTile - 1) / kTile;
        const int row0 = sg.rt * R;
        const __nv_bfloat16* qs = static_cast<const __nv_bfloat16*>(a.q) + static_cast<size_t>(sg.s) * a.n * a.q_stride;
        auto q_row = [&](int row) -> const __nv_bfloat16* {
            const int node = row / a.c.group;
            return qs + static_cast<size_t>(node) * a.q_stride + static_cast<size_t>(sg.h * a.c.group + row - node * a.c.group) * HD;
        };

        // queries as the right operand: lane (g, t) holds row g, 4 elements of each product
        uint32_t qf[NT][KS][2];
        float qmul[NT][2];                    // 2^-shift of rows 2t, 2t + 1, times scale and log2 e
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + 8 * nt + g;
            uint2 raw[KS];
            uint32_t amax = 0;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                raw[ks] = make_uint2(0, 0);
                if (row < p.rows) raw[ks] = *reinterpret_cast<const uint2*>(q_row(row) + 16 * (t + 4 * (ks >> 2)) + 4 * (ks & 3));
                amax = max(max(amax, raw[ks].x << 16 & 0x7fff0000u), max(raw[ks].x & 0x7fff0000u, max(raw[ks].y << 16 & 0x7fff0000u, raw[ks].y & 0x7fff0000u)));
            }
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            // 2^shift with the largest element at 2^14..2^15; a zero or non-finite row keeps its values
            const int e = static_cast<int>(amax >> 23) - 127;
            const int shift = amax == 0 || amax >= 0x7f800000u ? 0 : max(min(14 - e, 126), -113);
            const float up = __uint_as_float(static_cast<uint32_t>(shift + 127) << 23);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[nt][ks][0] = pack_f16(bf16_lo(raw[ks].x) * up, bf16_hi(raw[ks].x) * up);
                qf[nt][ks][1] = pack_f16(bf16_lo(raw[ks].y) * up, bf16_hi(raw[ks].y) * up);
            }
            const float down = __uint_as_float(static_cast<uint32_t>(127 - shift) << 23) * zscale;
            qmul[nt][0] = __shfl_sync(0xffffffffu, down, 8 * t);        // row 2t's lanes are 8t .. 8t + 3
            qmul[nt][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
        }

        float o[NT][MT][4], m[NT][2], sh[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = kLow, sh[nt][0] = sh[nt][1] = kLeastShift, l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
            for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.0f;
        }
        // m and sh of rows 2t, 2t + 1 for two groups of tokens: [group][row] the largest scores, log2 of the values' scale
        auto raise = [&](int nt, const float (&top)[2][2], const float (&lv)[2]) {
            float m2[2], kept[2], sh2[2];                               // kept: sh that leaves the numerators as they are
            bool any = false;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                m2[r] = fmaxf(m[nt][r], ceilf(fmaxf(top[0][r], top[1][r])));
                const float t2 = fmaxf(top[0][r] - m2[r] + lv[0], top[1][r] - m2[r] + lv[1]);
                kept[r] = sh[nt][r] - (m2[r] - m[nt][r]);
                sh2[r] = fmaxf(fmaxf(kept[r], ceilf(t2) - kHead), kLeastShift);
                any |= m2[r] > m[nt][r] || sh2[r] > kept[r];
            }
            if (!__any_sync(0xffffffffu, any)) return;
            const float f0 = ex2(kept[0] - sh2[0]), f1 = ex2(kept[1] - sh2[1]);
#pragma unroll
            for (int r = 0; r < 2; ++r) l[nt][r] *= ex2(m[nt][r] - m2[r]), m[nt][r] = m2[r], sh[nt][r] = sh2[r];
#pragma unroll
            for (int i = 0; i < MT; ++i) o[nt][i][0] *= f0, o[nt][i][1] *= f1, o[nt][i][2] *= f0, o[nt][i][3] *= f1;
        };
        // what takes a weight to P (2^126 at most: beyond it, a weight of less than 2^-112 takes less)
        auto to_p = [&](int nt, int r, float lv) { return ex2(fminf(lv - sh[nt][r], 126.0f)); };

        const int c_end = sg.t1 < cached_tiles ? sg.t1 : cached_tiles;
        if (sg.t0 < c_end) {
            Tokens<HD> next;
            int pid[2];
            int tok = sg.t0 * kTile + warp * kTok;
            page_ids(a, sg.s, tok, len, pid);
            next.load(a, pid, sg.h, tok, len);
            page_ids(a, sg.s, tok + kTile, sg.t0 + 1 < c_end ? len : 0, pid);
            for (int tile = sg.t0; tile < c_end; ++tile, tok += kTile) {
                Tokens<HD> cur = next;
                if (tile + 1 < c_end) {
                    next.load(a, pid, sg.h, tok + kTile, len);
                    page_ids(a, sg.s, tok + 2 * kTile, tile + 2 < c_end ? len : 0, pid);
                }
                if (cur.n[0] + cur.n[1] == 0) continue;
                const float lv[2] = {log2f(cur.vs[0]), log2f(cur.vs[1])};   // -inf: values of zeros
                float s[NT][2][4];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) s[nt][f][0] = s[nt][f][1] = s[nt][f][2] = s[nt][f][3] = 0.0f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        const uint32_t lo = cur.k[f][0][ks >> 2][ks & 3], hi = cur.k[f][1][ks >> 2][ks & 3];
                        const uint32_t a0 = widen2(lo), a1 = widen2(hi), a2 = widen2_hi(lo), a3 = widen2_hi(hi);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_f16(s[nt][f], a0, a1, a2, a3, qf[nt][ks][0], qf[nt][ks][1]);
                    }
                }
                uint32_t pf[NT][2][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float top[2][2];
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const float f0 = qmul[nt][0] * cur.ks[f], f1 = qmul[nt][1] * cur.ks[f];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const bool there = g + 8 * e < cur.n[f];
                            // (rounded, so that a large score cannot differ from its maximum)
                            s[nt][f][2 * e] = there ? __fmul_rn(s[nt][f][2 * e], f0) : -INFINITY;
                            s[nt][f][2 * e + 1] = there ? __fmul_rn(s[nt][f][2 * e + 1], f1) : -INFINITY;
                        }
                        top[f][0] = fmaxf(s[nt][f][0], s[nt][f][2]), top[f][1] = fmaxf(s[nt][f][1], s[nt][f][3]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) {
                            top[f][0] = fmaxf(top[f][0], __shfl_xor_sync(0xffffffffu, top[f][0], d));
                            top[f][1] = fmaxf(top[f][1], __shfl_xor_sync(0xffffffffu, top[f][1], d));
                        }
                    }
                    raise(nt, top, lv);
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const float up0 = to_p(nt, 0, lv[f]), up1 = to_p(nt, 1, lv[f]);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float w0 = ex2(s[nt][f][2 * e] - m[nt][0]), w1 = ex2(s[nt][f][2 * e + 1] - m[nt][1]);
                            l[nt][0] += w0, l[nt][1] += w1;
                            pf[nt][f][e] = transpose8(pack_f16(w0 * up0, w1 * up1));
                        }
                    }
                }
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int w = 0; w < Tokens<HD>::VW; ++w) {
                        // bytes b of tokens 2t, 2t + 1 side by side: elements 4w .. 4w + 3 of the lane
                        const uint32_t x01 = __byte_perm(cur.v[f][0][w], cur.v[f][1][w], 0x5140), x23 = __byte_perm(cur.v[f][0][w], cur.v[f][1][w], 0x7362);
                        const uint32_t y01 = __byte_perm(cur.v[f][2][w], cur.v[f][3][w], 0x5140), y23 = __byte_perm(cur.v[f][2][w], cur.v[f][3][w], 0x7362);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t xx = i ? x23 : x01, yy = i ? y23 : y01;
                            const uint32_t a0 = widen2(xx), a1 = widen2_hi(xx), a2 = widen2(yy), a3 = widen2_hi(yy);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][2 * w + i], a0, a1, a2, a3, pf[nt][f][0], pf[nt][f][1]);
                        }
                    }
            }
        }
        // the new tokens (at most as many as there are rows), one per warp and step, in fp32
        if (sg.t1 > cached_tiles) {
            const int j0 = (sg.t0 > cached_tiles ? sg.t0 - cached_tiles : 0) * kTile;
            const int j1 = min(a.n, (sg.t1 - cached_tiles) * kTile);
            for (int j = j0 + warp; j < j1; j += kWarps) {
                const size_t tokrow = static_cast<size_t>(sg.s) * a.n + j;
                const uint32_t* kp = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(a.k) + tokrow * a.k_stride +
                                                                       static_cast<size_t>(sg.h) * HD + EL * g);
                const uint32_t* vp = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(a.v) + tokrow * a.v_stride +
                                                                       static_cast<size_t>(sg.h) * HD + EL * g);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float z[2];
                    bool see[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = row0 + 8 * nt + 2 * t + e;
                        see[e] = row < p.rows && attn_sees(a, sg.s, row / a.c.group, j);
                        z[e] = 0.0f;
                        if (row < p.rows) {
                            const uint32_t* qp = reinterpret_cast<const uint32_t*>(q_row(row) + EL * g);
#pragma unroll
                            for (int d = 0; d < EL / 2; ++d) {
                                const uint32_t qw = qp[d], kw = kp[d];
                                z[e] = fmaf(bf16_lo(qw), bf16_lo(kw), fmaf(bf16_hi(qw), bf16_hi(kw), z[e]));
                            }
                        }
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) z[e] += __shfl_xor_sync(0xffffffffu, z[e], d);
                        z[e] = see[e] ? __fmul_rn(z[e], zscale) : -INFINITY;
                    }
                    if (!__any_sync(0xffffffffu, see[0] || see[1])) continue;
                    raise(nt, {{z[0], z[1]}, {-INFINITY, -INFINITY}}, {0.0f, 0.0f});
                    const float w0 = ex2(z[0] - m[nt][0]), w1 = ex2(z[1] - m[nt][1]);
                    // every lane of a row holds its weight; the sums are added over the lanes later
                    if (g == 0) l[nt][0] += w0, l[nt][1] += w1;
                    const float p0 = w0 * to_p(nt, 0, 0.0f), p1 = w1 * to_p(nt, 1, 0.0f);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const float v0 = bf16_lo(vp[i]), v1 = bf16_hi(vp[i]);
                        // an unseen token's value may be NaN
                        if (see[0]) o[nt][i][0] = fmaf(p0, v0, o[nt][i][0]), o[nt][i][2] = fmaf(p0, v1, o[nt][i][2]);
                        if (see[1]) o[nt][i][1] = fmaf(p1, v0, o[nt][i][1]), o[nt][i][3] = fmaf(p1, v1, o[nt][i][3]);
                    }
                }
            }
        }

        // join the warps
        __syncthreads();                                                // the item before has been read
        for (int rr = warp; rr < R && row0 + rr < p.rows; rr += kWarps) {
            const bool there = attn_row_present(a, sg.s, (row0 + rr) / a.c.group);
            if (lane == 0) present[rr] = there;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nt][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (g == 0) sml[warp][8 * nt + 2 * t + e] = make_float2(m[nt][e], sum), ssh[warp][8 * nt + 2 * t + e] = sh[nt][e];
                float* to = so[warp][8 * nt + 2 * t + e] + EL * g;
#pragma unroll
                for (int i = 0; i < MT; i += 2)
                    *reinterpret_cast<float4*>(to + 2 * i) = make_float4(o[nt][i][e], o[nt][i][2 + e], o[nt][i + 1][e], o[nt][i + 1][2 + e]);
            }
        }
        __syncthreads();
        const bool whole = sg.t0 == 0 && sg.t1 == sg.tiles;
        const int slot = attn_slot(blockIdx.x, sg.t0);
        for (int i = threadIdx.x; i < R * (HD / 4); i += 32 * kWarps) {
            const int rr = i / (HD / 4), d = 4 * (i - rr * (HD / 4)), row = row0 + rr;
            if (row >= p.rows) continue;
            const int node = row / a.c.group, head = sg.h * a.c.group + row - node * a.c.group;
            float mm = sml[0][rr].x, ll = 0.0f, top = -INFINITY, e[kWarps];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, sml[w][rr].x);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {                          // the numerators are a warp's times 2^e
                ll = fmaf(sml[w][rr].y, ex2(sml[w][rr].x - mm), ll);
                e[w] = ssh[w][rr] + (sml[w][rr].x - mm);
                top = fmaxf(top, e[w]);
            }
            float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = ex2(e[w] - top);
                const float4 ov = *reinterpret_cast<const float4*>(&so[w][rr][d]);
                v.x = fmaf(ov.x, f, v.x), v.y = fmaf(ov.y, f, v.y), v.z = fmaf(ov.z, f, v.z), v.w = fmaf(ov.w, f, v.w);
            }
            const bool none = !present[rr] || ll == 0.0f;
            const float inv = 1.0f / ll, half = ex2(0.5f * top);        // 2^top in two steps: it may pass fp32 where the output does not
            v.x = none ? 0.0f : v.x * inv * half * half, v.y = none ? 0.0f : v.y * inv * half * half;
            v.z = none ? 0.0f : v.z * inv * half * half, v.w = none ? 0.0f : v.w * inv * half * half;
            if (whole) {
                const size_t at = (static_cast<size_t>(sg.s) * a.n + node) * a.c.hq + head;
                const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
                uint2 w;
                w.x = *reinterpret_cast<const uint32_t*>(&lo), w.y = *reinterpret_cast<const uint32_t*>(&hi);
                *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at * HD + d) = w;
                if (a.lse && d == 0) a.lse[at] = none ? -INFINITY : (mm + log2f(ll)) * kLn2;
            } else {
                const size_t at = static_cast<size_t>(slot) * p.rt + rr;
                *reinterpret_cast<float4*>(p.part_o + at * HD + d) = v;
                if (d == 0) p.part_ml[at] = present[rr] ? make_float2(mm, ll) : make_float2(-INFINITY, 0.0f);
            }
        }
    }
}

}  // namespace

cudaError_t launch_attn_rows(cudaStream_t st, int num_sms, const AttnArgs& a, AttnSplit p) {
    p.tile_tokens = kTile;
    p.min_tiles = 1;
    const size_t smem = (static_cast<size_t>(a.c.b) + 1) * 8;
    auto run = [&](auto kernel, int nt, std::atomic<uint64_t>& done) {
        p.rt = 8 * nt;
        p.row_tiles = (p.rows + p.rt - 1) / p.rt;
        p.ctas = min(num_sms * 2, kAttnMaxCtas);
        attn_place_parts(a, &p);
        auto launch = [&] { return launch_pdl(kernel, dim3(p.ctas), dim3(32 * kWarps), smem, st, a, p); };
        // the list of many sequences needs more than the default
        const cudaError_t r = smem > 8 * 1024 ? launch_with_smem(kernel, (kMaxCacheBatch + 1) * 8, done, launch) : launch();
        return r != cudaSuccess ? r : launch_attn_combine(st, a, p);
    };
    static std::atomic<uint64_t> done[4];
    if (a.c.hd == 64) return p.rows <= 8 ? run(rows_attention_kernel<64, 1>, 1, done[0]) : run(rows_attention_kernel<64, 2>, 2, done[1]);
    return p.rows <= 8 ? run(rows_attention_kernel<128, 1>, 1, done[2]) : run(rows_attention_kernel<128, 2>, 2, done[3]);
}

}  // namespace tf
