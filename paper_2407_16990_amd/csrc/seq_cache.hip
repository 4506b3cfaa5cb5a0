// The paged cache of include/rh_seq.h: pages, block table and slots (rh_cache_plan), and the new keys and values into their slots
// (rh_cache_write).
#include "seq_common.h"

// ---------------------------------------------------------------------------------------------------------------
// rh_cache_plan
// ---------------------------------------------------------------------------------------------------------------
// Everything follows from running sums over the streams (at most 2048): the pages that ended streams give back, the pages
// and tokens asked for, and, once it is known who is granted, the pages taken and the tokens placed.  So every workgroup
// works the sums out for itself, in LDS - a few KB that come from the L2 - and then fills its share of the slots, of the table
// and of the stack; no second launch and no workgroup that waits for another.  The page at stack position p below the old
// height is in memory; above, it is one that this call puts there, and is found among the ended streams' table entries
// by bisection of their running sum, so that nothing that this launch writes is read by it.  Bound by latency: a call of 8 streams takes 4.9 us, where an empty
// launch takes 2.2 and lengths, scan and table entries are a way to memory each; 500 streams with chunks, 917 thousand slots, 8.8, of them 0.7 at a copy's rate.  The lengths and
// the height may be replaced in place: then the workgroup that finishes reading last (an atomic count) writes them, else the first.
#define PLAN_T 256
// Workgroups: one for every 512 slots, and for every 4096 pages of the table, of which ended streams may give back any number; at most
// four a CU.  500 streams with chunks (917 thousand slots): 15.1 us with one a CU, 11.9 with two, 10.4 with four or eight; 64 with
// chunks of 100: 13.6 with a workgroup for 1024 slots, 9.3 for 512.
#define PLAN_SLOTS 512
#define PLAN_PAGES 4096
#define PLAN_A_CU 4
#define PLAN_PER (RH_SEQ_MAX_STREAMS / PLAN_T)

struct plan_args {
    const int32_t *n_new, *lengths, *free_count;
    int32_t *table, *free_pages, *slots, *new_off, *new_lengths, *new_count;
    uint32_t* ticket;
    seq_div page;
    int32_t n_streams, n_pages, max_pages, n_slots;
};

// Exclusive running sums of a[0 .. N) over the workgroup's threads; `total`: the sums of all.  A thread's value is below 2^34 (eight
// of 31 bits): it goes as two words, the low one of 16 bits, whose sums over a wave stay within 32.
template <int N>
__device__ __forceinline__ void plan_scan(int64_t (&a)[N], int64_t (&total)[N], int64_t (*s_wave)[PLAN_T / 64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t v = ((int64_t)(uint32_t)seq_scan((int32_t)(a[i] >> 16)) << 16) + (uint32_t)seq_scan((int32_t)(a[i] & 0xFFFF));
        if (lane == 63) s_wave[i][wave] = v;
        a[i] = v - a[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        total[i] = 0;
#pragma unroll
        for (int w = 0; w < PLAN_T / 64; ++w) { if (w < wave) a[i] += s_wave[i][w]; total[i] += s_wave[i][w]; }
    }
    __syncthreads();
}

// Largest b in [0, n) with s[b] <= x; s ascending, s[0] <= x.
__device__ __forceinline__ int plan_find(const int32_t* s, int n, int32_t x)
{
    int lo = 0;
    for (int hi = n; hi - lo > 1;) { const int mid = (lo + hi) >> 1; if (s[mid] <= x) lo = mid; else hi = mid; }
    return lo;
}

__global__ __launch_bounds__(PLAN_T) void k_seq_plan(plan_args a)
{
    extern __shared__ int32_t s_mem[];                       // per stream: tokens placed before it, pages taken before it, pages given back before it, length
    __shared__ int64_t s_wave[3][PLAN_T / 64];
    __shared__ uint32_t s_last;
    const int B = a.n_streams, t = threadIdx.x, per = (B + PLAN_T - 1) / PLAN_T, b0 = t * per;
    const int page = (int)a.page.d;
    int32_t *s_off = s_mem, *s_start = s_off + B + 1, *s_back = s_start + B + 1, *s_old = s_back + B + 1;
    int32_t height = *a.free_count;
    height = height < 0 ? 0 : height > a.n_pages ? a.n_pages : height;

    int32_t old[PLAN_PER], ask[PLAN_PER], need[PLAN_PER];    // ask < 0: ended; need: pages asked for, of an ended stream pages given back; -1: do not fit the row
    int64_t sum[3] = {0, 0, 0}, total[3];
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int b = b0 + i;
        old[i] = ask[i] = need[i] = 0;
        if (i >= per || b >= B) continue;
        const int32_t n = a.n_new[b], len = a.lengths[b];
        old[i] = len < 0 ? 0 : len;
        ask[i] = n;
        const uint32_t row = (uint32_t)a.max_pages * page;   // at most 2^31 - 1 - page
        const int32_t have = (uint32_t)old[i] <= row ? (int32_t)seq_quot((uint32_t)old[i] + page - 1, a.page) : a.max_pages;
        if (n < 0) {
            need[i] = have;
            sum[0] += have;
        } else if ((uint32_t)old[i] + (uint32_t)n <= row) {
            need[i] = (int32_t)seq_quot((uint32_t)old[i] + (uint32_t)n + page - 1, a.page) - have;
            sum[1] += need[i]; sum[2] += n;
        } else need[i] = -1;
    }
    plan_scan(sum, total, s_wave);
    const int64_t returned = total[0], top = height + returned;
    int64_t back = sum[0], upto = sum[1], tokens = sum[2], got[2] = {0, 0}, placed[2];
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int b = b0 + i;
        if (i >= per || b >= B) continue;
        s_back[b] = (int32_t)back;
        s_old[b] = old[i];
        if (ask[i] < 0) { back += need[i]; need[i] = 0; old[i] = 0; ask[i] = 0; continue; }
        bool ok = need[i] >= 0;
        if (ok) {
            upto += need[i]; tokens += ask[i];
            ok = (need[i] == 0 || upto <= top) && tokens <= a.n_slots;
        }
        if (!ok) { need[i] = 0; ask[i] = 0; }
        got[0] += ask[i]; got[1] += need[i];
    }
    plan_scan(got, placed, s_wave);
    int32_t off = (int32_t)got[0], start = (int32_t)got[1];
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int b = b0 + i;
        if (i >= per || b >= B) continue;
        s_off[b] = off; s_start[b] = start;
        off += ask[i]; start += need[i];
    }
    if (t == 0) { s_off[B] = (int32_t)placed[0]; s_start[B] = (int32_t)placed[1]; s_back[B] = (int32_t)returned; }
    __syncthreads();

    // the page at stack position p < top
    auto stacked = [&](int32_t p) -> int32_t {
        if (p < height) return a.free_pages[p];
        const int32_t r = p - height;
        const int b = plan_find(s_back, B, r);
        return a.table[(size_t)b * a.max_pages + (r - s_back[b])];
    };
    const int id = blockIdx.x * PLAN_T + t, stride = gridDim.x * PLAN_T;
    const int32_t n_tok = (int32_t)placed[0], n_taken = (int32_t)placed[1], high = (int32_t)top - 1;
    // pages that come back from the last thread on, pages taken from the middle, slots from the first: mostly no workgroup has to do with two of them
    for (int r = stride - 1 - id; r < (int32_t)returned; r += stride) {
        const int b = plan_find(s_back, B, r);
        if (height + r < a.n_pages) a.free_pages[height + r] = a.table[(size_t)b * a.max_pages + (r - s_back[b])];
    }
    for (int i = id < stride / 2 ? id + (stride + 1) / 2 : id - stride / 2; i < n_taken; i += stride) {
        const int b = plan_find(s_start, B, i);
        const int have = (int)seq_quot((uint32_t)(s_old[b] + page - 1), a.page);
        a.table[(size_t)b * a.max_pages + have + (i - s_start[b])] = stacked(high - i);
    }
    // slots: four neighbours a thread, which mostly share stream and page
    for (int64_t first = (int64_t)id * 4; first < a.n_slots; first += (int64_t)stride * 4) {
        int b = first < n_tok ? plan_find(s_off, B, (int32_t)first) : B, have = 0, last = -1;
        int32_t p = 0, slot[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int32_t i = (int32_t)first + e;            // n_slots < 2^31 - 4
            slot[e] = -1;
            if (i >= n_tok) continue;
            while (i >= s_off[b + 1]) { ++b; last = -1; }    // i is below the last stream's end
            const uint32_t pos = (uint32_t)(s_old[b] + (i - s_off[b]));
            const int k = (int)seq_quot(pos, a.page);
            if (k != last) {
                have = (int)seq_quot((uint32_t)(s_old[b] + page - 1), a.page);
                p = k < have ? a.table[(size_t)b * a.max_pages + k] : stacked(high - s_start[b] - (k - have));
                last = k;
            }
            slot[e] = p * page + (int32_t)(pos - (uint32_t)k * page);
        }
        if (first + 4 <= a.n_slots) seq_store(a.slots + first, u32x4{(uint32_t)slot[0], (uint32_t)slot[1], (uint32_t)slot[2], (uint32_t)slot[3]});
        else for (int e = 0; first + e < a.n_slots; ++e) a.slots[first + e] = slot[e];
    }
    // what is replaced in place is written by the last workgroup to have read it
    if (!a.ticket) { if (blockIdx.x) return; }
    else {
        if (t == 0) s_last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        __syncthreads();
        if (!s_last) return;
        if (t == 0) *a.ticket = 0;
    }
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int b = b0 + i;
        if (i >= per || b >= B) continue;
        a.new_lengths[b] = old[i] + ask[i];
        a.new_off[b] = s_off[b];
    }
    if (t == 0) { a.new_off[B] = n_tok; *a.new_count = (int32_t)top - n_taken; }
}

rh_status rh_launch_cache_plan(rh_ctx* ctx, plan_args& a)
{
    const int64_t wgs = (int64_t)a.n_slots / PLAN_SLOTS + (int64_t)a.n_streams * a.max_pages / PLAN_PAGES;
    const int grid = (int)(wgs < 1 ? 1 : wgs < PLAN_A_CU * ctx->n_cu ? wgs : PLAN_A_CU * ctx->n_cu);
    if (grid > 1 && (a.new_lengths == a.lengths || a.new_count == a.free_count)) {
        const rh_status st = seq_counters(ctx);
        if (st != RH_OK) return st;
        a.ticket = ctx->seq_cnt;
    }
    hipLaunchKernelGGL(k_seq_plan, dim3(grid), dim3(PLAN_T), 4 * (size_t)(a.n_streams + 1) * sizeof(int32_t), ctx->stream, a);
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}

extern "C" rh_status rh_cache_plan(rh_ctx* ctx, const int32_t* n_new, const int32_t* lengths, int32_t n_streams, int32_t page,
                                   int32_t n_pages, int32_t max_pages, int32_t* block_table, int32_t* free_pages,
                                   const int32_t* free_count, int32_t* slots, int32_t n_slots, int32_t* new_off,
                                   int32_t* new_lengths, int32_t* new_count)
{
    if (!ctx) return RH_E_INVALID;
    if (n_streams < 1 || n_streams > RH_SEQ_MAX_STREAMS)
        RH_FAIL(ctx, RH_E_CAPACITY, "rh_cache_plan: %d streams outside [1,%d]", n_streams, RH_SEQ_MAX_STREAMS);
    if (page < 1 || n_pages < 1 || max_pages < 1 || n_slots < 1 || n_slots > 0x7FFFFFF0)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_plan: page=%d, n_pages=%d, max_pages=%d, n_slots=%d must be positive (and n_slots below 2^31 - 16)", page, n_pages, max_pages, n_slots);
    if ((int64_t)page * n_pages > 0x7FFFFFFFll || (int64_t)page * max_pages > 0x7FFFFFFFll - page)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_plan: %d pages (%d a stream) of %d tokens pass 2^31 slots", n_pages, max_pages, page);
    // whatever the lengths claim, ended streams give back no more pages than the table has entries: positions on the stack stay within 32 bits
    if ((int64_t)n_streams * max_pages + n_pages > 0x7FFFFFFFll)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_plan: %d rows of %d pages and a stack of %d pass 2^31 entries", n_streams, max_pages, n_pages);
    if (!n_new || !lengths || !block_table || !free_pages || !free_count || !slots || !new_off || !new_lengths || !new_count)
        RH_FAIL(ctx, RH_E_INVALID, "rh_cache_plan: null argument");
    plan_args a = {n_new, lengths, free_count, block_table, free_pages, slots, new_off, new_lengths, new_count, nullptr,
                   seq_make_div((uint32_t)page), n_streams, n_pages, max_pages, n_slots};
    return rh_launch_cache_plan(ctx, a);
}

// ---------------------------------------------------------------------------------------------------------------
// rh_cache_write
// ---------------------------------------------------------------------------------------------------------------
// Bound by memory: every key and value read and written once (27600 tokens of 8 heads of 128, bf16 to e4m3: 171 MB in 39 to 45 us, 3.8 to 4.4 TB/s; half the
// bytes written go to scattered slots, a quarter of a KB at a time).  G lanes (a power of two) take a head's row, eight elements each, so
// that the largest magnitude is a few lane exchanges; lanes past the head's size idle.
// Rows a thread, whose loads are in flight together: two where they are quantised (27600 tokens of 8 heads of 128, with quotients not yet corrected: 44.1 us, one row
// 48.7, four 47.1), else one (bf16 46.0, two 48.2; 64 tokens 2.2 and 2.4).
template <typename C> constexpr int write_rows() { return sizeof(C) == 1 ? 2 : 1; }

struct write_args {
    const void* src[2];
    int64_t src_stride[2][2];
    void* dst[2];
    float* scale[2];
    int64_t dst_stride[2][3];
    const int32_t* slots;
    seq_div page, heads;
    int64_t rows;            // n * heads
    int32_t dim, n_slots;
};

template <typename T> __device__ __forceinline__ void write_load(const T* p, float (&x)[8]);
template <> __device__ __forceinline__ void write_load<float>(const float* p, float (&x)[8])
{
    const f32x4 a = seq_load<f32x4>(p), b = seq_load<f32x4>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
template <> __device__ __forceinline__ void write_load<__bf16>(const __bf16* p, float (&x)[8])
{
    const uint4 u = seq_load<uint4>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = seq_bf16_lo(w[i]); x[2 * i + 1] = seq_bf16_hi(w[i]); }
}

template <typename T, typename C, int G>
__global__ __launch_bounds__(256) void k_seq_write(write_args a)
{
    constexpr int WRITE_ROWS = write_rows<C>(), R = 256 / G; // R: rows of a workgroup at a time
    const int kv = blockIdx.y, g = threadIdx.x & (G - 1), d = g * 8;
    const bool in = d < a.dim;
    const int64_t first = (int64_t)blockIdx.x * (R * WRITE_ROWS) + threadIdx.x / G;
    uint32_t tok[WRITE_ROWS], head[WRITE_ROWS];
    int32_t slot[WRITE_ROWS];
    float x[WRITE_ROWS][8];
#pragma unroll
    for (int i = 0; i < WRITE_ROWS; ++i) {
        const uint32_t row = (uint32_t)(first + i * R < a.rows ? first + i * R : 0);
        tok[i] = seq_quot(row, a.heads); head[i] = row - tok[i] * a.heads.d;
        slot[i] = first + i * R < a.rows ? a.slots[tok[i]] : -1;
    }
#pragma unroll
    for (int i = 0; i < WRITE_ROWS; ++i)                     // rows that are none read row 0
        write_load((const T*)a.src[kv] + (int64_t)tok[i] * a.src_stride[kv][0] + head[i] * a.src_stride[kv][1] + (in ? d : 0), x[i]);
#pragma unroll
    for (int i = 0; i < WRITE_ROWS; ++i) {
        if (slot[i] < 0 || slot[i] >= a.n_slots) continue;   // the same for a group's lanes
        const uint32_t p = seq_quot((uint32_t)slot[i], a.page), line = (uint32_t)slot[i] - p * a.page.d;
        const int64_t at = p * a.dst_stride[kv][0] + line * a.dst_stride[kv][1] + head[i] * a.dst_stride[kv][2] + d;
        const float(&v)[8] = x[i];
        if constexpr (sizeof(C) == 1) {
            float most = 0.f;
            if (in) {
#pragma unroll
                for (int e = 0; e < 8; ++e) most = v[e] != v[e] ? v[e] : fabsf(v[e]) > most ? fabsf(v[e]) : most;     // a NaN stays
            }
#pragma unroll
            for (int o = G / 2; o; o >>= 1) { const float u = __shfl_xor(most, o); most = u != u || u > most ? u : most; }
            most = most < SEQ_AMAX_MIN ? SEQ_AMAX_MIN : most;
            const seq_scale scale = seq_make_scale(most);
            if (g == 0) a.scale[kv][((int64_t)p * a.heads.d + head[i]) * a.page.d + line] = scale.value;
            const uint2 q = make_uint2(seq_pack_scaled(v[0], v[1], v[2], v[3], scale), seq_pack_scaled(v[4], v[5], v[6], v[7], scale));
            // past the L2, where the scales' lines, of which each store fills a word, then stay until they are full (44.3 -> 42.8 us)
            if (in) __builtin_nontemporal_store((uint64_t)q.y << 32 | q.x, (uint64_t*)((uint8_t*)a.dst[kv] + at));
        } else if constexpr (sizeof(C) == 2) {
            uint4 q;
            q.x = seq_pack_bf16(v[0], v[1]); q.y = seq_pack_bf16(v[2], v[3]); q.z = seq_pack_bf16(v[4], v[5]); q.w = seq_pack_bf16(v[6], v[7]);
            if (in) *(uint4*)((__bf16*)a.dst[kv] + at) = q;
        } else if (in) {
            float* o = (float*)a.dst[kv] + at;
            *(f32x4*)o = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4*)(o + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    }
}

template <typename T, typename C>
static void launch_write(hipStream_t s, const write_args& a)
{
    constexpr int WRITE_ROWS = write_rows<C>();
    const int lanes = a.dim / 8;
#define W(G) hipLaunchKernelGGL((k_seq_write<T, C, G>), dim3((unsigned)((a.rows + 256 / G * WRITE_ROWS - 1) / (256 / G * WRITE_ROWS)), 2), dim3(256), 0, s, a)
    if (lanes <= 4) W(4); else if (lanes <= 8) W(8); else if (lanes <= 16) W(16); else W(32);
#undef W
}

extern "C" rh_status rh_cache_write(rh_ctx* ctx, const rh_kv_cache* cache, const void* k, const int64_t k_stride[2], const void* v,
                                    const int64_t v_stride[2], int32_t type, const int32_t* slots, int32_t n)
{
    if (!ctx) return RH_E_INVALID;
    if (!cache || !k_stride || !v_stride || (n && (!k || !v || !slots))) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_write: null argument");
    if (type != RH_T_F32 && type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_write: values of type %d", type);
    const rh_status st = seq_check_cache(ctx, "rh_cache_write", cache);
    if (st != RH_OK) return st;
    if (type == RH_T_BF16 && cache->type == RH_T_F32) RH_FAIL(ctx, RH_E_UNIMPLEMENTED, "rh_cache_write: bf16 values into an fp32 cache");
    if (n < 0 || (int64_t)n * cache->heads > 0x7FFFFFFFll) RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_write: %d tokens of %d heads", n, cache->heads);
    if (n == 0) return RH_OK;
    write_args a;
    a.src[0] = k; a.src[1] = v; a.dst[0] = cache->k; a.dst[1] = cache->v; a.scale[0] = cache->k_scale; a.scale[1] = cache->v_scale;
    for (int i = 0; i < 2; ++i) { a.src_stride[0][i] = k_stride[i]; a.src_stride[1][i] = v_stride[i]; }
    for (int i = 0; i < 3; ++i) { a.dst_stride[0][i] = cache->k_stride[i]; a.dst_stride[1][i] = cache->v_stride[i]; }
    a.slots = slots; a.page = seq_make_div((uint32_t)cache->page); a.heads = seq_make_div((uint32_t)cache->heads);
    a.rows = (int64_t)n * cache->heads; a.dim = cache->dim; a.n_slots = cache->n_pages * cache->page;
    if (type == RH_T_BF16) {
        if (cache->type == RH_T_BF16) launch_write<__bf16, __bf16>(ctx->stream, a); else launch_write<__bf16, uint8_t>(ctx->stream, a);
    } else {
        if (cache->type == RH_T_F32) launch_write<float, float>(ctx->stream, a);
        else if (cache->type == RH_T_BF16) launch_write<float, __bf16>(ctx->stream, a);
        else launch_write<float, uint8_t>(ctx->stream, a);
    }
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}

rh_status seq_check_cache(rh_ctx* ctx, const char* name, const rh_kv_cache* c)
{
    if (c->type != RH_T_F32 && c->type != RH_T_BF16 && c->type != RH_T_E4M3) RH_FAIL(ctx, RH_E_INVALID, "%s: a cache of type %d", name, c->type);
    if (!c->k || !c->v) RH_FAIL(ctx, RH_E_INVALID, "%s: null cache", name);
    if ((c->type == RH_T_E4M3) != (c->k_scale != nullptr) || (c->type == RH_T_E4M3) != (c->v_scale != nullptr))
        RH_FAIL(ctx, RH_E_INVALID, "%s: scales belong to an e4m3 cache, and only to one", name);
    if (c->n_pages < 1 || c->page < 1 || (int64_t)c->n_pages * c->page > 0x7FFFFFFFll)
        RH_FAIL(ctx, RH_E_SHAPE, "%s: %d pages of %d tokens", name, c->n_pages, c->page);
    if (c->heads < 1 || c->dim < 32 || c->dim > RH_SEQ_MAX_DIM || c->dim % 32)
        RH_FAIL(ctx, RH_E_SHAPE, "%s: %d heads of %d elements (a multiple of 32 up to %d)", name, c->heads, c->dim, RH_SEQ_MAX_DIM);
    const int64_t whole = c->type == RH_T_F32 ? 4 : c->type == RH_T_BF16 ? 8 : 16;       // elements of 16 bytes
    for (int i = 0; i < 3; ++i)
        if (c->k_stride[i] < 0 || c->v_stride[i] < 0 || c->k_stride[i] % whole || c->v_stride[i] % whole)
            RH_FAIL(ctx, RH_E_SHAPE, "%s: cache strides must be multiples of 16 bytes and not negative", name);
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) RH_FAIL(ctx, RH_E_INVALID, "%s: the cache must be 16-byte aligned", name);
    return RH_OK;
}

__global__ void k_seq_zero(uint32_t* p, uint32_t n)
{
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0;
}

// Both are made once, at their full size, at the first call that wants them: what a graph has recorded stays where it is.  Not while the stream is being captured, where the
// fill of the counters would only be recorded, and calls ahead of the first replay would count from whatever is there.
static rh_status seq_may_allocate(rh_ctx* ctx)
{
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(ctx->stream, &capture);
    if (e == hipErrorStreamCaptureImplicit || (e == hipSuccess && capture != hipStreamCaptureStatusNone))
        RH_FAIL(ctx, RH_E_STATE, "the sequence operators' memory is not there yet and cannot be allocated in a stream capture: make one such call before it");
    return RH_OK;
}

rh_status seq_counters(rh_ctx* ctx)
{
    if (ctx->seq_cnt) return RH_OK;
    const rh_status st = seq_may_allocate(ctx);
    if (st != RH_OK) return st;
    const uint32_t n = (uint32_t)SEQ_ROWS(ctx);
    uint32_t* made = nullptr;
    if (hipMalloc((void**)&made, n * sizeof(uint32_t)) != hipSuccess) RH_FAIL(ctx, RH_E_NOMEM, "%u counters", n);
    // The context has them once they are zero: the next call may be on another stream, and one behind a lost fill would trust them.
    hipLaunchKernelGGL(k_seq_zero, dim3((n + 255) / 256), dim3(256), 0, ctx->stream, made, n);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = hipStreamSynchronize(ctx->stream);
    if (e != hipSuccess) { (void)hipFree(made); RH_FAIL(ctx, RH_E_DEVICE, "clearing counters: %s", hipGetErrorString(e)); }
    ctx->seq_cnt = made;
    return RH_OK;
}

rh_status seq_scratch(rh_ctx* ctx)
{
    if (ctx->seq_ws) return RH_OK;
    const rh_status st = seq_may_allocate(ctx);
    if (st != RH_OK) return st;
    const size_t bytes = (size_t)SEQ_ROWS(ctx) * SEQ_ROW_BYTES(RH_SEQ_MAX_DIM);
    if (hipMalloc(&ctx->seq_ws, bytes) != hipSuccess) { ctx->seq_ws = nullptr; RH_FAIL(ctx, RH_E_NOMEM, "scratch memory of %zu bytes", bytes); }
    return RH_OK;
}
