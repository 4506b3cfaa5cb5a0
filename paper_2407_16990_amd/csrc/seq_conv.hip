// rh_state_conv: short causal convolution along the tokens of every stream, a channel at a time.
//
// Bound by memory: every input is read once and every output written once (past the L2: 58 -> 52 us below); the width - 1 inputs ahead of a thread's rows are read again (30 streams of
// 920 rows, 2048 channels in bf16, inputs that no cache holds: 227 MB and 23 read twice in 51 us, 4.4 TB/s).
// A thread has 16 bytes of channels and a run of rows, whose last inputs it keeps in registers.  Runs begin where streams do,
// so that only a stream's first run looks at its state, and that thread, once it has read it, writes the state behind the last row:
// no other thread writes it, and it may be replaced in place.  The last piece of a row that is no multiple of one is loaded from further ahead, with channels of the thread before, which may
// have replaced them by then: row_place leaves them out, and has to.
#include "seq_rows.h"
#include "seq_streams.h"

#define CONV_BATCH 4             // rows whose loads are in flight together, while the four ahead are worked on (eight: 57 for 51 us, see below)

struct conv_args {
    streams_args r;
    const void* x;
    const float *weight, *bias;
    void *state, *y;
    int64_t x_stride, y_stride;
    seq_div pieces;              // threads a row
    int32_t channels, silu, run, log_run;
    bool past;
};

template <typename T, int W>
struct conv_taps {
    static constexpr int E = 16 / sizeof(T);
    float w[W][E], bias[E];
    __device__ __forceinline__ void load(const conv_args& a, int c)
    {
        auto get = [&](const float* p, float (&v)[E]) {
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                float u[4];
                row_place<float, 4>(row_load<float, 4>(p, c + e, a.channels), c + e, a.channels, u);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[e + k] = u[k];
            }
        };
#pragma unroll
        for (int j = 0; j < W; ++j) get(a.weight + (int64_t)j * a.channels, w[j]);
        if (a.bias) get(a.bias, bias);
        else
#pragma unroll
            for (int e = 0; e < E; ++e) bias[e] = 0.f;
    }
    // the output whose W inputs begin at v[0]
    template <int N> __device__ __forceinline__ void apply(const float (&v)[N][E], int first, bool silu, float (&y)[E]) const
    {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float s = bias[e];
#pragma unroll
            for (int j = 0; j < W; ++j) s = fmaf(w[j][e], v[first + j][e], s);
            y[e] = silu ? seq_silu(s) : s;
        }
    }
};

// One row a stream.
template <typename T, int W>
__global__ __launch_bounds__(256) void k_seq_conv_step(conv_args a)
{
    constexpr int E = 16 / sizeof(T);
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;
    const int b = (int)seq_quot(id, a.pieces), c = (int)(id - (uint32_t)b * a.pieces.d) * E;
    if (b >= a.r.n_rows) return;
    const int32_t from = streams_slot(a.r, b), to = streams_into(a.r, b);
    const T* old = (const T*)a.state + (int64_t)(from < 0 ? 0 : from) * (W - 1) * a.channels;
    u32x4 in[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) in[j] = from < 0 ? u32x4{0, 0, 0, 0} : row_load<T, E>(old + (int64_t)j * a.channels, c, a.channels);
    in[W - 1] = row_load<T, E>((const T*)a.x + b * a.x_stride, c, a.channels);
    conv_taps<T, W> taps;
    taps.load(a, c);
    float v[W][E], y[E];
#pragma unroll
    for (int j = 0; j < W; ++j) row_place<T, E>(in[j], c, a.channels, v[j]);
    taps.apply(v, 0, a.silu, y);
    row_store<T, E>((T*)a.y + b * a.y_stride + c, a.channels - c, y);
    if (to < 0) return;
    T* kept = (T*)a.state + (int64_t)to * (W - 1) * a.channels + c;
#pragma unroll
    for (int j = 1; j < W; ++j) row_store<T, E>(kept + (int64_t)(j - 1) * a.channels, a.channels - c, v[j]);
}

// Any number of rows a stream.
template <typename T, int W>
__global__ __launch_bounds__(STREAMS_T) void k_seq_conv(conv_args a)
{
    constexpr int E = 16 / sizeof(T);
    extern __shared__ int32_t s_first[];                     // of more than 64 streams: runs of the streams before
    __shared__ int32_t s_wave[STREAMS_T / 64];
    const uint32_t id = blockIdx.x * STREAMS_T + threadIdx.x;
    const int q = (int)seq_quot(id, a.pieces), c = (int)(id - (uint32_t)q * a.pieces.d) * E;
    conv_taps<T, W> taps;
    taps.load(a, c);                                         // on their way while the run is looked for
    auto runs = [&](int32_t n) { return (int32_t)(((uint32_t)n + a.run - 1) >> a.log_run); };
    int32_t begin, end, all;
    int32_t row;
    int b;
    if (a.r.n_streams <= 64) {
        streams_lane s;
        if (!streams_few(a.r, runs, s, all)) return;
        b = 0;
#pragma unroll
        for (int step = 32; step; step >>= 1) {
            const int32_t ahead = __shfl(s.before, b + step);               // every lane of the wave takes part
            if (b + step < a.r.n_streams && ahead <= q) b += step;
        }
        begin = __shfl(s.begin, b); end = __shfl(s.end, b);
        row = begin + (q - __shfl(s.before, b)) * a.run;
        if (q >= all) return;
    } else {
        if (!streams_sums(a.r, s_first, s_wave, runs) || q >= s_first[a.r.n_streams]) return;
        b = streams_find(s_first, a.r.n_streams, q);
        streams_rows(a.r, b, begin, end);
        row = begin + (q - s_first[b]) * a.run;
    }
    const int32_t stop = end - row < a.run ? end : row + a.run;
    const T* x = (const T*)a.x;

    float v[W - 1 + CONV_BATCH][E];
    if (row > begin) {                                       // a run is W - 1 rows or more: they are all the stream's
        u32x4 in[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) in[j] = row_load<T, E>(x + (int64_t)(row - (W - 1) + j) * a.x_stride, c, a.channels);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) row_place<T, E>(in[j], c, a.channels, v[j]);
    } else {
        const int32_t from = streams_slot(a.r, b), to = streams_into(a.r, b);
        const T* old = (const T*)a.state + (int64_t)(from < 0 ? 0 : from) * (W - 1) * a.channels;
        u32x4 in[W - 1], last[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            in[j] = from < 0 ? u32x4{0, 0, 0, 0} : row_load<T, E>(old + (int64_t)j * a.channels, c, a.channels);
            const int32_t at = end - begin - (W - 1) + j;    // below 0: an input of the state that stays
            last[j] = at >= 0 ? row_load<T, E>(x + (int64_t)(begin + at) * a.x_stride, c, a.channels)
                      : from < 0 ? u32x4{0, 0, 0, 0} : row_load<T, E>(old + (int64_t)(at + W - 1) * a.channels, c, a.channels);
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) row_place<T, E>(in[j], c, a.channels, v[j]);
        if (to >= 0) {
            T* kept = (T*)a.state + (int64_t)to * (W - 1) * a.channels + c;
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                float u[E];
                row_place<T, E>(last[j], c, a.channels, u);
                row_store<T, E>(kept + (int64_t)j * a.channels, a.channels - c, u);
            }
        }
    }
    const T* px = x + (int64_t)row * a.x_stride;
    T* py = (T*)a.y + (int64_t)row * a.y_stride + c;
    const bool whole = a.channels - c >= E;
    u32x4 in[CONV_BATCH];
    auto load = [&](int rows) __attribute__((always_inline)) {               // rows that are left
#pragma unroll
        for (int i = 0; i < CONV_BATCH; ++i) in[i] = row_load<T, E>(px + (i < rows ? i : rows - 1) * a.x_stride, c, a.channels);
        px += CONV_BATCH * a.x_stride;
    };
    load(stop - row);
    for (int32_t t = row; t < stop; t += CONV_BATCH) {
        const int rows = stop - t;
#pragma unroll
        for (int i = 0; i < CONV_BATCH; ++i) row_place<T, E>(in[i], c, a.channels, v[W - 1 + i]);
        if (rows > CONV_BATCH) load(rows - CONV_BATCH);      // while these are worked on
#pragma unroll
        for (int i = 0; i < CONV_BATCH; ++i) {
            float y[E];
            taps.apply(v, i, a.silu, y);
            if (i < rows) row_store<T, E>(py + i * a.y_stride, whole ? E : a.channels - c, y, a.past);
        }
        py += CONV_BATCH * a.y_stride;
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) v[j][e] = v[CONV_BATCH + j][e];
    }
}

template <typename T, int W>
static void launch_conv(rh_ctx* ctx, conv_args& a)
{
    if (!a.r.offsets) {
        const int64_t threads = (int64_t)a.r.n_rows * a.pieces.d;
        hipLaunchKernelGGL((k_seq_conv_step<T, W>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, ctx->stream, a);
        return;
    }
    const int64_t threads = ((int64_t)a.r.n_rows / a.run + a.r.n_streams) * a.pieces.d;       // as many runs as any offsets give
    hipLaunchKernelGGL((k_seq_conv<T, W>), dim3((unsigned)((threads + STREAMS_T - 1) / STREAMS_T)), dim3(STREAMS_T), a.r.n_streams > 64 ? (a.r.n_streams + 1) * sizeof(int32_t) : 0, ctx->stream, a);
}
template <typename T>
static void launch_conv(rh_ctx* ctx, conv_args& a, int width)
{
    switch (width) {
    case 2: return launch_conv<T, 2>(ctx, a);
    case 3: return launch_conv<T, 3>(ctx, a);
    case 4: return launch_conv<T, 4>(ctx, a);
    case 5: return launch_conv<T, 5>(ctx, a);
    case 6: return launch_conv<T, 6>(ctx, a);
    case 7: return launch_conv<T, 7>(ctx, a);
    default: return launch_conv<T, 8>(ctx, a);
    }
}

rh_status streams_check(rh_ctx* ctx, const char* name, const rh_state_rows* r, streams_args* a)
{
    if (r->n_streams < 0 || r->n_rows < 0 || r->n_slots < 0 || r->n_rows > 0x7FFF0000) RH_FAIL(ctx, RH_E_SHAPE, "%s: %d rows of %d streams, %d slots", name, r->n_rows, r->n_streams, r->n_slots);
    if (r->n_streams && !r->slots) RH_FAIL(ctx, RH_E_INVALID, "%s: null argument", name);
    if (!r->offsets && r->n_rows != r->n_streams) RH_FAIL(ctx, RH_E_SHAPE, "%s: %d rows of %d streams without offsets", name, r->n_rows, r->n_streams);
    if (r->offsets && r->n_streams > RH_SEQ_MAX_STREAMS)
        RH_FAIL(ctx, RH_E_CAPACITY, "%s: %d streams with offsets, more than %d", name, r->n_streams, RH_SEQ_MAX_STREAMS);
    *a = {r->offsets, r->slots, r->into ? r->into : r->slots, r->past, r->n_streams, r->n_rows, r->n_slots};
    return RH_OK;
}

extern "C" rh_status rh_state_conv(rh_ctx* ctx, const rh_state_rows* rows, const void* x, int64_t x_stride, const float* weight,
                                   const float* bias, int32_t type, int32_t channels, int32_t width, int32_t silu, void* state,
                                   void* y, int64_t y_stride)
{
    if (!ctx) return RH_E_INVALID;
    if (!rows || !weight) RH_FAIL(ctx, RH_E_INVALID, "rh_state_conv: null argument");
    conv_args a;
    const rh_status st = streams_check(ctx, "rh_state_conv", rows, &a.r);
    if (st != RH_OK) return st;
    if (type != RH_T_F32 && type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_state_conv: rows of type %d", type);
    if (channels < 1 || channels > 0x7FFFFFFF - 16) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_conv: %d channels", channels);
    if (width < 2 || width > RH_SEQ_MAX_TAPS) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_conv: a width of %d (2 to %d)", width, RH_SEQ_MAX_TAPS);
    if (x_stride < channels || y_stride < channels) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_conv: a row stride below %d", channels);
    if (rows->n_rows == 0 || rows->n_streams == 0) return RH_OK;
    if (!x || !y || (rows->n_slots && !state)) RH_FAIL(ctx, RH_E_INVALID, "rh_state_conv: null argument");
    const int E = type == RH_T_F32 ? 4 : 8, pieces = (channels + E - 1) / E;
    // Rows a run: 16, and 8 where that would be fewer than two workgroups a CU.  8, 16, 32 and 64 of them, us, inputs that no cache holds: 30 streams of 920, 2048 channels in bf16 54, 51,
    // 59 and 53 (32 leave three workgroups and a half a CU); 37 of up to 1500, 515 in fp32 29.3, 26.4, 29.1 and 40.5.
    a.log_run = ((int64_t)rows->n_rows >> 4) * pieces < (int64_t)ctx->n_cu * 2 * STREAMS_T ? 3 : 4;
    a.run = 1 << a.log_run;
    if ((rows->offsets ? (int64_t)rows->n_rows / a.run + rows->n_streams : rows->n_rows) * pieces > 0x7FFFF000ll)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_state_conv: %d rows of %d channels", rows->n_rows, channels);
    a.x = x; a.weight = weight; a.bias = bias; a.state = state; a.y = y; a.x_stride = x_stride; a.y_stride = y_stride;
    a.pieces = seq_make_div((uint32_t)pieces); a.channels = channels; a.silu = silu != 0;
    a.past = (int64_t)rows->n_rows * channels * (type == RH_T_F32 ? 4 : 2) >= ROWS_PAST;
    if (type == RH_T_F32) launch_conv<float>(ctx, a, width); else launch_conv<__bf16>(ctx, a, width);
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}
