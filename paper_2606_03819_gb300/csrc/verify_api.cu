// C ABI of the verifier's side (declared in include/treeflash.h): argument checks and launches. No allocation and no
// state between calls.
#include <math.h>

#include "verify.cuh"

namespace {

using namespace tf;

tf_status check_cache(const tf_cache_dims* dims, CacheShape* o) {
    if (!dims) return TF_ERR_INVALID_ARG;
    const tf_cache_dims& d = *dims;
    if (d.batch < 1 || d.heads < 1 || d.kv_heads < 1 || d.head_dim < 1 || d.page < 1 || d.n_pages < 1 || d.max_pages < 1)
        return TF_ERR_INVALID_ARG;
    if (d.dtype != TF_BF16 && d.dtype != TF_F32) return TF_ERR_INVALID_ARG;
    if (d.heads % d.kv_heads != 0) return TF_ERR_INVALID_ARG;
    if (d.batch > kMaxCacheBatch || d.heads > 1024) return TF_ERR_UNSUPPORTED;
    if (d.head_dim % 16 != 0 || d.head_dim > kMaxHeadDim) return TF_ERR_UNSUPPORTED;
    int log2 = 0;
    while ((1 << log2) < d.page && log2 < 8) ++log2;
    if ((1 << log2) != d.page || d.page < 16 || d.page > 128) return TF_ERR_UNSUPPORTED;
    // Slots (page * tokens + place) and places in a sequence are int32. The attention kernels round a sequence's length up to
    // their tiles and look up to two tiles of 128 tokens ahead, which has to fit too.
    const long long top = (1ll << 31) - 1, longest = (1ll << 31) - 1024;
    if (static_cast<long long>(d.n_pages) * d.page > top || static_cast<long long>(d.max_pages) * d.page > longest)
        return TF_ERR_UNSUPPORTED;
    *o = CacheShape{d.batch, d.heads, d.kv_heads, d.heads / d.kv_heads, d.head_dim, d.page, log2, d.n_pages, d.max_pages,
                    d.dtype};
    return TF_OK;
}

bool aligned(const void* p, size_t n) { return p && reinterpret_cast<uintptr_t>(p) % n == 0; }

// Rows of new tokens: 16-byte aligned, a row's elements contiguous.
bool rows_ok(const CacheShape& c, const void* p, long long stride, int heads) {
    const int esize = c.dtype == TF_BF16 ? 2 : 4;
    return aligned(p, 16) && stride >= static_cast<long long>(heads) * c.hd && stride <= (1ll << 31) && stride * esize % 16 == 0;
}

bool caches_ok(const void* k, const void* v, const float* ks, const float* vs) {
    return aligned(k, 16) && aligned(v, 16) && aligned(ks, 4) && aligned(vs, 4);
}

tf_status sm_count(int* sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return TF_ERR_CUDA;
    if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || *sms < 1) return TF_ERR_CUDA;
    return TF_OK;
}

tf_status done(cudaError_t e) { return e == cudaSuccess ? TF_OK : TF_ERR_CUDA; }

// New tokens of one call: their rows (n * group) and the pieces of work stay within 31 bits.
tf_status check_new_tokens(const CacheShape& c, int n) {
    if (n < 1) return TF_ERR_INVALID_ARG;
    if (n > (1 << 20) || static_cast<long long>(n) * c.group > (1 << 24)) return TF_ERR_UNSUPPORTED;
    if (static_cast<long long>(c.b) * c.hkv * (static_cast<long long>(n) * c.group + 128) > (1ll << 31) - 1)
        return TF_ERR_UNSUPPORTED;
    return TF_OK;
}

}  // namespace

extern "C" {

tf_status tf_cache_plan(const tf_cache_dims* dims, const tf_plan_args* args, tf_stream_t stream) {
    CacheShape c;
    const tf_status s = check_cache(dims, &c);
    if (s != TF_OK) return s;
    if (!args) return TF_ERR_INVALID_ARG;
    const tf_plan_args& p = *args;
    if (!aligned(p.seq_len, 4) || !aligned(p.delta, 4) || !aligned(p.block_table, 4) || !aligned(p.free_list, 4) ||
        !aligned(p.free_count, 4) || !aligned(p.new_len, 4) || !aligned(p.dev_status, 4))
        return TF_ERR_INVALID_ARG;
    if (p.slot_map && (!aligned(p.slot_map, 4) || p.width < 1)) return TF_ERR_INVALID_ARG;
    return done(launch_cache_plan(reinterpret_cast<cudaStream_t>(stream), c, p));
}

tf_status tf_cache_append(const tf_cache_dims* dims, const tf_append_args* args, tf_stream_t stream) {
    CacheShape c;
    const tf_status s = check_cache(dims, &c);
    if (s != TF_OK) return s;
    if (!args) return TF_ERR_INVALID_ARG;
    const tf_append_args& p = *args;
    if (p.n_rows < 1 || p.width < 1) return TF_ERR_INVALID_ARG;
    if (!rows_ok(c, p.k, p.k_stride, c.hkv) || !rows_ok(c, p.v, p.v_stride, c.hkv)) return TF_ERR_INVALID_ARG;
    if (!aligned(p.slot_map, 4) || (p.src && !aligned(p.src, 4)) || !aligned(p.dev_status, 4)) return TF_ERR_INVALID_ARG;
    if (!caches_ok(p.k_cache, p.v_cache, p.k_scale, p.v_scale)) return TF_ERR_INVALID_ARG;
    return done(launch_cache_append(reinterpret_cast<cudaStream_t>(stream), c, p));
}

tf_status tf_attention_workspace_size(const tf_cache_dims* dims, int32_t n, size_t* bytes) {
    CacheShape c;
    tf_status s = check_cache(dims, &c);
    if (s == TF_OK) s = bytes ? check_new_tokens(c, n) : TF_ERR_INVALID_ARG;
    if (s != TF_OK) return s;
    *bytes = attention_ws_bytes(c, n);
    return TF_OK;
}

tf_status tf_tree_attention(const tf_cache_dims* dims, const tf_attention_args* args, tf_stream_t stream) {
    AttnArgs a;
    tf_status s = check_cache(dims, &a.c);
    if (s == TF_OK) s = args ? check_new_tokens(a.c, args->n) : TF_ERR_INVALID_ARG;
    if (s != TF_OK) return s;
    const tf_attention_args& p = *args;
    if (!rows_ok(a.c, p.q, p.q_stride, a.c.hq) || !rows_ok(a.c, p.k, p.k_stride, a.c.hkv) || !rows_ok(a.c, p.v, p.v_stride, a.c.hkv))
        return TF_ERR_INVALID_ARG;
    if (!caches_ok(p.k_cache, p.v_cache, p.k_scale, p.v_scale) || !aligned(p.block_table, 4) || !aligned(p.seq_len, 4) ||
        !aligned(p.out, 16) || (p.lse && !aligned(p.lse, 4)) || !aligned(p.dev_status, 4))
        return TF_ERR_INVALID_ARG;
    if (!(p.scale > 0.0f) || !isfinite(p.scale)) return TF_ERR_INVALID_ARG;
    if (!aligned(p.ws, 256) || p.ws_bytes < attention_ws_bytes(a.c, p.n)) return TF_ERR_WORKSPACE;
    int sms = 0;
    s = sm_count(&sms);
    if (s != TF_OK) return s;
    a.n = p.n;
    a.q = p.q, a.k = p.k, a.v = p.v, a.q_stride = p.q_stride, a.k_stride = p.k_stride, a.v_stride = p.v_stride;
    a.k_cache = static_cast<const uint8_t*>(p.k_cache), a.v_cache = static_cast<const uint8_t*>(p.v_cache);
    a.k_scale = p.k_scale, a.v_scale = p.v_scale, a.table = p.block_table, a.seq_len = p.seq_len;
    a.mask = p.mask, a.scale = p.scale, a.out = p.out, a.lse = p.lse, a.status = p.dev_status, a.ws = p.ws;
    return done(launch_tree_attention(reinterpret_cast<cudaStream_t>(stream), sms, a));
}

tf_status tf_sample(const tf_sample_args* args, tf_stream_t stream) {
    if (!args) return TF_ERR_INVALID_ARG;
    const tf_sample_args& p = *args;
    if (p.rows < 1 || p.V < 1 || p.rows_per_seq < 1 || p.row_stride < p.V) return TF_ERR_INVALID_ARG;
    if (p.dtype != TF_BF16 && p.dtype != TF_F32) return TF_ERR_INVALID_ARG;
    if (p.V > (1 << 20)) return TF_ERR_UNSUPPORTED;
    if (!aligned(p.logits, p.dtype == TF_BF16 ? 2 : 4) || !aligned(p.u, 4) || !aligned(p.tok, 4)) return TF_ERR_INVALID_ARG;
    if ((p.temperature && !aligned(p.temperature, 4)) || (p.top_k && !aligned(p.top_k, 4)) || (p.top_p && !aligned(p.top_p, 4)) ||
        (p.min_p && !aligned(p.min_p, 4)) || (p.logp && !aligned(p.logp, 4)))
        return TF_ERR_INVALID_ARG;
    int sms = 0;
    const tf_status s = sm_count(&sms);
    if (s != TF_OK) return s;
    return done(launch_sample(reinterpret_cast<cudaStream_t>(stream), sms, p));
}

}  // extern "C"
