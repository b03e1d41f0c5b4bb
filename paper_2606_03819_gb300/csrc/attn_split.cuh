// How the attention kernels share out their work, and the layout of partial results.
//
// The work of one item (sequence, head of keys, tile of query rows) is its tiles of tokens: the cached ones, then the
// new ones. Contexts are ragged and only the GPU knows them, so every CTA lists the tiles of all items from seq_len and
// takes an equal run of them: a long context is cut wherever a CTA's share ends, and a CTA may do several short ones.
// An item that lies in one CTA's run is finished there; the pieces of the others (at most two per CTA: the end of one
// item, the beginning of another) go to the workspace and a second kernel joins them, in the order of the tokens, so
// results do not depend on timing.
#pragma once

#include "verify.cuh"

namespace tf {

struct AttnSplit {
    int rows;          // query rows of one (sequence, head of keys): n * group
    int row_tiles;     // ceil(rows / RT)
    int tile_tokens;   // tokens per tile
    int min_tiles;     // least share of a CTA, in tiles
    int ctas;          // CTAs that share the work
    int rt;            // rows per tile (of partial results)
    float* part_o;     // [2 * ctas][rt][hd]: a piece's own output (numerators / sum), 0 where a row saw nothing of it
    float2* part_ml;   // [2 * ctas][rt]: of its scores in the base-2 log domain, m (the maximum or little more) and the sum of exp2(z - m)
};

__device__ __forceinline__ int attn_len(const AttnArgs& a, int s) {
    const int cap = a.c.max_pages << a.c.page_log2;   // 2^31 - 1024 at most: what follows may round it up and look ahead
    return min(max(a.seq_len[s], 0), cap);
}

// Tiles of every item of sequence s.
__device__ __forceinline__ int attn_tiles(const AttnArgs& a, const AttnSplit& p, int s) {
    return (attn_len(a, s) + p.tile_tokens - 1) / p.tile_tokens + (a.n + p.tile_tokens - 1) / p.tile_tokens;
}

// Exclusive prefix over the sequences of their tiles in prefix[0..b], by the calling warp.
__device__ __forceinline__ void attn_list(const AttnArgs& a, const AttnSplit& p, long long* prefix) {
    const int lane = threadIdx.x & 31;
    const int per_seq = a.c.hkv * p.row_tiles;
    long long run = 0;
    for (int s0 = 0; s0 < a.c.b; s0 += 32) {
        const int s = s0 + lane;
        const long long v = s < a.c.b ? static_cast<long long>(attn_tiles(a, p, s)) * per_seq : 0;
        long long incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (s < a.c.b) prefix[s] = run + incl - v;
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) prefix[a.c.b] = run;
}

__device__ __forceinline__ long long attn_share(const AttnSplit& p, long long total) {
    const long long even = (total + p.ctas - 1) / p.ctas;
    return even > p.min_tiles ? even : p.min_tiles;
}

// The sequence whose tiles hold tile x (every sequence has at least one: n >= 1).
__device__ __forceinline__ int attn_find(const long long* prefix, int b, long long x) {
    int lo = 0, hi = b - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (prefix[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

struct Segment {
    int s, h, rt, t0, t1, tiles;   // tiles t0..t1-1 of the item's `tiles`
};
__device__ __forceinline__ Segment attn_segment(const AttnArgs& a, const AttnSplit& p, const long long* prefix, long long x,
                                                long long end) {
    Segment g;
    g.s = attn_find(prefix, a.c.b, x);
    g.tiles = attn_tiles(a, p, g.s);
    const long long local = x - prefix[g.s];
    const int item = static_cast<int>(local / g.tiles);
    g.t0 = static_cast<int>(local - static_cast<long long>(item) * g.tiles);
    const long long left = end - x;
    g.t1 = g.tiles - g.t0 < left ? g.tiles : g.t0 + static_cast<int>(left);
    g.h = item / p.row_tiles;
    g.rt = item - g.h * p.row_tiles;
    return g;
}
// Where a piece of an item goes: 2c for one that does not hold the item's first tile, else 2c + 1.
__device__ __forceinline__ int attn_slot(int cta, int t0) { return 2 * cta + (t0 == 0 ? 1 : 0); }

// A row that its mask leaves empty sees nothing at all. The whole warp calls it for one node.
__device__ __forceinline__ bool attn_row_present(const AttnArgs& a, int s, int node) {
    if (a.mask == nullptr) return true;
    const uint8_t* m = a.mask + (static_cast<size_t>(s) * a.n + node) * a.n;
    bool any = false;
    for (int j = threadIdx.x & 31; j < a.n; j += 32) any |= m[j] != 0;
    return __any_sync(0xffffffffu, any);
}
__device__ __forceinline__ bool attn_sees(const AttnArgs& a, int s, int node, int j) {
    if (j >= a.n) return false;
    return a.mask ? a.mask[(static_cast<size_t>(s) * a.n + node) * a.n + j] != 0 : j <= node;
}

// CTAs that share the work, at most: the room of the partial results is laid out for this many whatever the GPU has.
constexpr int kAttnMaxCtas = 608;

// The room of the partial results in the workspace, for tiles of p->rt rows.
inline size_t attn_part_bytes(int rt, int hd) {
    return static_cast<size_t>(2) * kAttnMaxCtas * rt * (static_cast<size_t>(hd) * 4 + 8) + 256;
}
inline void attn_place_parts(const AttnArgs& a, AttnSplit* p) {
    uint8_t* ws = static_cast<uint8_t*>(a.ws);
    p->part_ml = reinterpret_cast<float2*>(ws);
    p->part_o = reinterpret_cast<float*>(ws + (static_cast<size_t>(2) * p->ctas * p->rt * 8 + 255) / 256 * 256);
}

// many rows per head (attn_tiles.cu)
bool attn_tiles_take(const CacheShape&);
size_t attn_tiles_ws_bytes(const CacheShape&, int n);
cudaError_t launch_attn_tiles(cudaStream_t, int num_sms, const AttnArgs&);
// few rows (attn_rows.cu)
cudaError_t launch_attn_rows(cudaStream_t, int num_sms, const AttnArgs&, AttnSplit);
cudaError_t launch_attn_combine(cudaStream_t, const AttnArgs&, const AttnSplit&);

}  // namespace tf
