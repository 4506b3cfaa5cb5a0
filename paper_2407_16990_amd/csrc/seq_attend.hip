// rh_cache_attend: attention of one new token of every stream over a paged cache.
#include "seq_common.h"

struct attend_args {
    const void *k, *v, *q;
    const float *k_scale, *v_scale;
    int64_t ks[3], vs[3], qs[2];
    const int32_t *table, *lengths;
    void* out;
    float* lse;
    seq_div page;
    int32_t n_pages, heads, q_heads, group, dim, max_pages, n_streams, window;
    float scale;
};

// One workgroup a stream and query head: scores of 256 tokens at a time, a token a thread, then their values, an element a thread.
template <typename T, typename C>
__global__ __launch_bounds__(256) void k_seq_attend(attend_args a)
{
    __shared__ float s_q[RH_SEQ_MAX_DIM], s_p[256], s_red[256];
    __shared__ int64_t s_at[256];
    const int b = blockIdx.y, h = blockIdx.x, kvh = h / a.group, t = threadIdx.x;
    int64_t len = a.lengths[b];
    const int64_t row = (int64_t)a.max_pages * a.page.d;
    len = len < 0 ? 0 : len > row ? row : len;
    const int64_t begin = a.window && len > a.window ? len - a.window : 0;
    if (t < a.dim) s_q[t] = seq_to_f32(((const T*)a.q)[b * a.qs[0] + h * a.qs[1] + t]);
    __syncthreads();
    float top = -INFINITY, total = 0.f, acc = 0.f;
    for (int64_t first = begin; first < len; first += 256) {
        const int64_t pos = first + t;
        float s = -INFINITY;
        s_at[t] = -1;
        float vscale = 1.f;
        if (pos < len) {
            const uint32_t k = seq_quot((uint32_t)pos, a.page), line = (uint32_t)pos - k * a.page.d;
            const int32_t p = a.table[(int64_t)b * a.max_pages + k];
            if (p >= 0 && p < a.n_pages) {
                const C* key = (const C*)a.k + p * a.ks[0] + line * a.ks[1] + kvh * a.ks[2];
                float dot = 0.f;
                for (int d = 0; d < a.dim; ++d) dot += s_q[d] * seq_to_f32(key[d]);
                if constexpr (sizeof(C) == 1) {
                    const int64_t at = ((int64_t)p * a.heads + kvh) * a.page.d + line;
                    dot *= a.k_scale[at];
                    vscale = a.v_scale[at];
                }
                s = dot * a.scale;
                s_at[t] = p * a.vs[0] + line * a.vs[1] + kvh * a.vs[2];
            }
        }
        s_red[t] = s;
        __syncthreads();
        for (int o = 128; o; o >>= 1) { if (t < o) s_red[t] = fmaxf(s_red[t], s_red[t + o]); __syncthreads(); }
        const float now = fmaxf(top, s_red[0]);
        __syncthreads();
        const float base = now == -INFINITY ? 0.f : now, fade = expf(top - base), p = expf(s - base);
        s_p[t] = p * vscale;
        s_red[t] = p;
        __syncthreads();
        for (int o = 128; o; o >>= 1) { if (t < o) s_red[t] += s_red[t + o]; __syncthreads(); }
        total = total * fade + s_red[0];
        acc *= fade;
        top = now;
        if (t < a.dim)
            for (int i = 0; i < 256; ++i) if (s_at[i] >= 0) acc += s_p[i] * seq_to_f32(((const C*)a.v)[s_at[i] + t]);
        __syncthreads();
    }
    const int64_t o = (int64_t)b * a.q_heads + h;
    if (t < a.dim) ((T*)a.out)[o * a.dim + t] = (T)(total > 0.f ? acc / total : total != total ? total : 0.f);
    if (t == 0 && a.lse) a.lse[o] = total > 0.f ? top + logf(total) : total != total ? total : -INFINITY;
}

extern "C" rh_status rh_cache_attend(rh_ctx* ctx, const rh_kv_cache* cache, const void* q, const int64_t q_stride[2], int32_t type,
                                     int32_t q_heads, const int32_t* block_table, int32_t max_pages, const int32_t* lengths,
                                     int32_t n_streams, float scale, int32_t window, void* out, float* lse)
{
    if (!ctx) return RH_E_INVALID;
    if (!cache || !q || !q_stride || !block_table || !lengths || !out) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: null argument");
    if (type != RH_T_F32 && type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: queries of type %d", type);
    const rh_status st = seq_check_cache(ctx, "rh_cache_attend", cache);
    if (st != RH_OK) return st;
    if ((type == RH_T_F32) != (cache->type == RH_T_F32))
        RH_FAIL(ctx, RH_E_UNIMPLEMENTED, "rh_cache_attend: queries of type %d over a cache of type %d", type, cache->type);
    if (q_heads < 1 || q_heads % cache->heads) RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_attend: %d query heads over %d of the cache", q_heads, cache->heads);
    if (n_streams < 1 || n_streams > RH_SEQ_MAX_STREAMS)
        RH_FAIL(ctx, RH_E_CAPACITY, "rh_cache_attend: %d streams outside [1,%d]", n_streams, RH_SEQ_MAX_STREAMS);
    if (max_pages < 1 || (int64_t)max_pages * cache->page > 0x7FFFFFFFll - cache->page)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_attend: %d pages of %d tokens a stream", max_pages, cache->page);
    if ((int64_t)q_heads * n_streams > 0x7FFFFFFFll / RH_SEQ_MAX_DIM) RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_attend: %d heads of %d streams", q_heads, n_streams);
    if (window < 0) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: a window of %d", window);
    if ((uintptr_t)out & 15) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: out must be 16-byte aligned");
    attend_args a;
    a.k = cache->k; a.v = cache->v; a.q = q; a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
    for (int i = 0; i < 3; ++i) { a.ks[i] = cache->k_stride[i]; a.vs[i] = cache->v_stride[i]; }
    for (int i = 0; i < 2; ++i) a.qs[i] = q_stride[i];
    a.table = block_table; a.lengths = lengths; a.out = out; a.lse = lse; a.page = seq_make_div((uint32_t)cache->page);
    a.n_pages = cache->n_pages; a.heads = cache->heads; a.q_heads = q_heads; a.group = q_heads / cache->heads; a.dim = cache->dim;
    a.max_pages = max_pages; a.n_streams = n_streams; a.window = window; a.scale = scale;
    const dim3 grid(q_heads, n_streams);
    if (cache->type == RH_T_F32) hipLaunchKernelGGL((k_seq_attend<float, float>), grid, dim3(256), 0, ctx->stream, a);
    else if (cache->type == RH_T_BF16) hipLaunchKernelGGL((k_seq_attend<__bf16, __bf16>), grid, dim3(256), 0, ctx->stream, a);
    else hipLaunchKernelGGL((k_seq_attend<__bf16, uint8_t>), grid, dim3(256), 0, ctx->stream, a);
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}
