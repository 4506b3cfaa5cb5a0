// rh_norm_residual: residual addition, root-mean-square norm, and the norm's output in 8 bits.
//
// Bound by memory: x and the residual are read once, the sum, y and its 8-bit form written once.  A row stays in the
// registers of the waves that own it: the mean square, and then the largest |y|, are sums and maxima over them.
// A row belongs to one wave where it is short, so that a workgroup of four waves needs no barrier, or to a part of one where it is shorter still.
// 14720 x 4095 of fp32, all outputs: 183 us, 5.6 TB/s; of bf16 126, 4.3 TB/s (rows at odd addresses; 4092: 108, 5.0 TB/s); 8 x 1024 of
// bf16, 8-bit output, 3.7, hardly more than an empty launch and a way to memory.
#include "seq_rows.h"

struct norm_args {
    const void *x, *residual;
    const float* weight;
    void *sum, *y;
    uint8_t* y8;
    float* y8_scale;
    int64_t x_stride, residual_stride, sum_stride;
    int32_t rows, cols;
    float eps;
};

// The sum (MAX: the largest, a NaN staying) of a value of every thread of a row's WAVES waves, or of its LANES lanes.
template <int WAVES, int LANES, bool MAX>
__device__ __forceinline__ float norm_over(float v, float* s_part)
{
    auto both = [](float a, float b) { return MAX ? (b != b || b > a ? b : a) : a + b; };
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v = both(v, __shfl_xor(v, o));
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s_part[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = both(v, s_part[w]);
        __syncthreads();
    }
    return v;
}

// a row's WAVES waves, of one of them LANES lanes, with ITEMS pieces a thread
template <typename T, int WAVES, int LANES, int ITEMS>
__global__ __launch_bounds__(WAVES > 1 ? WAVES * 64 : 256) void k_seq_norm(norm_args a)
{
    constexpr int E = 16 / sizeof(T), NT = WAVES * LANES, PER = WAVES > 1 ? 1 : 256 / LANES;       // threads a row, rows a workgroup
    __shared__ float s_part[WAVES > 1 ? WAVES * PER : 1];
    const int t = threadIdx.x % NT, sub = threadIdx.x / NT;
    const int row = blockIdx.x * PER + sub;
    if (PER > 1 && row >= a.rows) return;                    // PER > 1 only where a row is one wave's or less: no barrier is left behind
    const T* x = (const T*)a.x + row * a.x_stride;
    const T* r = (const T*)a.residual + row * a.residual_stride;
    float v[ITEMS][E], square = 0.f;
    u32x4 in[ITEMS], add[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) in[i] = row_load<T, E>(x, (t + i * NT) * E, a.cols);
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) add[i] = row_load<T, E>(r, (t + i * NT) * E, a.cols);
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) row_place<T, E>(in[i], (t + i * NT) * E, a.cols, v[i]);
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float u[E];
            row_place<T, E>(add[i], (t + i * NT) * E, a.cols, u);
#pragma unroll
            for (int e = 0; e < E; ++e) v[i][e] += u[e];
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) square += v[i][e] * v[i][e];
    square = norm_over<WAVES, LANES, false>(square, s_part);
    if (a.sum) {
        T* s = (T*)a.sum + row * a.sum_stride;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (t + i * NT) * E, n = a.cols - c;
            if (n > 0) row_store<T, E>(s + c, n, v[i]);
        }
    }
    if (!a.y && !a.y8) return;
    const float scale = 1.f / sqrtf(square / (float)a.cols + a.eps);
    float most = 0.f;
    constexpr int AHEAD = ITEMS < 4 ? ITEMS : 4;             // items whose weights are in flight
#pragma unroll
    for (int i0 = 0; i0 < ITEMS; i0 += AHEAD) {
        u32x4 weight[AHEAD][E / 4];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int e = 0; e < E; e += 4) weight[i][e / 4] = row_load<float, 4>(a.weight, (t + (i0 + i) * NT) * E + e, a.cols);
#pragma unroll
        for (int i = i0; i < i0 + AHEAD; ++i) {
            const int c = (t + i * NT) * E, n = a.cols - c;
            float w[E];
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                float u[4];
                row_place<float, 4>(weight[i - i0][e / 4], c + e, a.cols, u);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[e + k] = u[k];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[i][e] = v[i][e] * scale * w[e];
                const float m = fabsf(v[i][e]);
                most = m != m || m > most ? m : most;
            }
            if (a.y && n > 0) row_store<T, E>((T*)a.y + (int64_t)row * a.cols + c, n, v[i]);
        }
    }
    if (!a.y8) return;
    most = norm_over<WAVES, LANES, true>(most, s_part);
    most = most < SEQ_AMAX_MIN ? SEQ_AMAX_MIN : most;
    const seq_scale y8_scale = seq_make_scale(most);
    if (t == 0) a.y8_scale[row] = y8_scale.value;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (t + i * NT) * E, n = a.cols - c;
        if (n <= 0) continue;
        uint8_t* o = a.y8 + (int64_t)row * a.cols + c;
        u32x4 q = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < E; e += 4) q[e / 4] = seq_pack_scaled(v[i][e], v[i][e + 1], v[i][e + 2], v[i][e + 3], y8_scale);
        if (n < E) row_put<1>(o, n, q);
        else if constexpr (E == 8) seq_store(o, make_uint2(q[0], q[1]));
        else seq_store(o, q[0]);
    }
}

template <typename T>
static void launch_norm(hipStream_t s, const norm_args& a)
{
    constexpr int E = 16 / sizeof(T);
    const int pieces = (a.cols + E - 1) / E;                 // of 16 bytes, one a thread and item
#define N(WAVES, LANES, ITEMS) hipLaunchKernelGGL((k_seq_norm<T, WAVES, LANES, ITEMS>), dim3(WAVES > 1 ? a.rows : (a.rows + 256 / LANES - 1) / (256 / LANES)), \
                                                  dim3(WAVES > 1 ? WAVES * 64 : 256), 0, s, a)
    // Short rows share a wave (16050 rows of 60, fp32: 10.7 -> 5.9 us, of 200 in bf16 13.3 -> 10.0).
    if (pieces <= 8) N(1, 8, 1);
    else if (pieces <= 16) N(1, 16, 1);
    else if (pieces <= 32) N(1, 32, 1);
    else if (pieces <= 64) N(1, 64, 1);
    // Two pieces a thread while a workgroup's waves last.  8 rows of 1800 in bf16: 4.7 us, with four a thread in one wave 6.3, with one a thread 4.4; 14720 of 1024 in fp32
    // 43.5, 43.5, 47.5; 1000 of 4095 in fp32 13.5, 13.6, 16.7.  A single row of 8000 in bf16 4.9, 5.8, 5.3.
    else if (pieces <= 128) N(1, 64, 2);
    else if (pieces <= 256) N(2, 64, 2);
    else if (pieces <= 512) N(4, 64, 2);
    else if (pieces <= 1024) N(8, 64, 2);
    else if (pieces <= 2048) N(8, 64, 4);
    else if (pieces <= 4096) N(16, 64, 4);
    else if constexpr (E == 4) N(16, 64, 8);                     // of bf16 none is that long
#undef N
}

extern "C" rh_status rh_norm_residual(rh_ctx* ctx, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                                      const float* weight, int32_t type, int32_t n_rows, int32_t n_cols, float eps, void* sum,
                                      int64_t sum_stride, void* y, uint8_t* y8, float* y8_scale)
{
    if (!ctx) return RH_E_INVALID;
    if (!weight || (n_rows && !x)) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_residual: null argument");
    if (n_rows && !y8 != !y8_scale) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_residual: 8-bit output and its scales go together");
    if (n_rows && !sum && !y && !y8) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_residual: no output asked for");
    if (type != RH_T_F32 && type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_residual: rows of type %d", type);
    if (n_rows < 0 || n_cols < 1 || n_cols > RH_SEQ_MAX_COLS)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_norm_residual: %d rows of %d elements (1 to %d)", n_rows, n_cols, RH_SEQ_MAX_COLS);
    if (x_stride < n_cols || (residual && residual_stride < n_cols) || (sum && sum_stride < n_cols))
        RH_FAIL(ctx, RH_E_SHAPE, "rh_norm_residual: a row stride below %d", n_cols);
    if (!(eps >= 0.f)) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_residual: eps must not be negative");
    if (n_rows == 0) return RH_OK;
    const norm_args a = {x, residual, weight, sum, y, y8, y8_scale, x_stride, residual_stride, sum_stride, n_rows, n_cols, eps};
    if (type == RH_T_F32) launch_norm<float>(ctx->stream, a); else launch_norm<__bf16>(ctx->stream, a);
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}
