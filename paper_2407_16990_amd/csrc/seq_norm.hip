// rh_norm_residual: residual addition, root-mean-square norm, and the norm's output in 8 bits.
//
// Bound by memory: x and the residual are read once, the sum, y and its 8-bit form written once.  A row stays in the
// registers of the waves that own it: the mean square, and then the largest |y|, are sums and maxima over them.
// A row belongs to one wave where it is short, so that a workgroup of four waves needs no barrier.
#include "seq_common.h"

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

// E elements (16 bytes) from a row that may start at any element; `n` of them exist.
template <typename T, int E>
__device__ __forceinline__ void norm_load(const T* p, int n, float (&v)[E])
{
    if (n >= E) {
        if constexpr (sizeof(T) == 2) {
            const uint4 u = seq_load<uint4>(p);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = seq_bf16_lo(w[i]); v[2 * i + 1] = seq_bf16_hi(w[i]); }
        } else {
            const f32x4 a = seq_load<f32x4>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = i < n ? seq_to_f32(p[i]) : 0.f;
    }
}

template <typename T, int E>
__device__ __forceinline__ void norm_store(T* p, int n, const float (&v)[E])
{
    if (n >= E) {
        if constexpr (sizeof(T) == 2) {
            uint4 u;
            u.x = seq_pack_bf16(v[0], v[1]); u.y = seq_pack_bf16(v[2], v[3]); u.z = seq_pack_bf16(v[4], v[5]); u.w = seq_pack_bf16(v[6], v[7]);
            seq_store(p, u);
        } else seq_store(p, f32x4{v[0], v[1], v[2], v[3]});
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) if (i < n) p[i] = (T)v[i];
    }
}

// The sum (MAX: the largest, a NaN staying) of a value of every thread of a row's WAVES waves.
template <int WAVES, bool MAX>
__device__ __forceinline__ float norm_over(float v, float* s_part)
{
    auto both = [](float a, float b) { return MAX ? (b != b || b > a ? b : a) : a + b; };
#pragma unroll
    for (int o = 32; o; o >>= 1) v = both(v, __shfl_xor(v, o));
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

template <typename T, int WAVES, int ITEMS>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void k_seq_norm(norm_args a)
{
    constexpr int E = 16 / sizeof(T), NT = WAVES * 64, PER = WAVES > 4 ? 1 : 4 / WAVES;       // threads a row, rows a workgroup
    __shared__ float s_part[WAVES > 1 ? WAVES * PER : 1];
    const int t = threadIdx.x % NT, sub = threadIdx.x / NT;
    const int row = blockIdx.x * PER + sub;
    if (PER > 1 && row >= a.rows) return;                    // PER > 1 only where a row is one wave's: no barrier is left behind
    const T* x = (const T*)a.x + row * a.x_stride;
    const T* r = (const T*)a.residual + row * a.residual_stride;
    float v[ITEMS][E], square = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (t + i * NT) * E, n = a.cols - c;
        if (n > 0) norm_load<T, E>(x + c, n, v[i]);
        else { for (int e = 0; e < E; ++e) v[i][e] = 0.f; }
    }
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (t + i * NT) * E, n = a.cols - c;
            if (n <= 0) continue;
            float u[E];
            norm_load<T, E>(r + c, n, u);
#pragma unroll
            for (int e = 0; e < E; ++e) v[i][e] += u[e];
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) square += v[i][e] * v[i][e];
    square = norm_over<WAVES, false>(square, s_part);
    if (a.sum) {
        T* s = (T*)a.sum + row * a.sum_stride;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (t + i * NT) * E, n = a.cols - c;
            if (n > 0) norm_store<T, E>(s + c, n, v[i]);
        }
    }
    if (!a.y && !a.y8) return;
    const float scale = 1.f / sqrtf(square / (float)a.cols + a.eps);
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (t + i * NT) * E, n = a.cols - c;
        if (n <= 0) continue;
        float w[E];
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            float u[4];
            norm_load<float, 4>(a.weight + c + e, n - e, u);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[e + k] = u[k];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[i][e] = v[i][e] * scale * w[e];
            const float m = fabsf(v[i][e]);
            most = m != m || m > most ? m : most;
        }
        if (a.y) norm_store<T, E>((T*)a.y + (int64_t)row * a.cols + c, n, v[i]);
    }
    if (!a.y8) return;
    most = norm_over<WAVES, true>(most, s_part);
    most = most < SEQ_AMAX_MIN ? SEQ_AMAX_MIN : most;
    const float inv = SEQ_E4M3_MAX / most;
    if (t == 0) a.y8_scale[row] = most / SEQ_E4M3_MAX;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (t + i * NT) * E, n = a.cols - c;
        if (n <= 0) continue;
        uint8_t* o = a.y8 + (int64_t)row * a.cols + c;
        uint32_t q[E / 4];
#pragma unroll
        for (int e = 0; e < E; e += 4) q[e / 4] = seq_pack_e4m3(v[i][e] * inv, v[i][e + 1] * inv, v[i][e + 2] * inv, v[i][e + 3] * inv);
        if (n >= E) {
            if constexpr (E == 8) seq_store(o, make_uint2(q[0], q[1])); else seq_store(o, q[0]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (e < n) o[e] = (uint8_t)(q[e / 4] >> (8 * (e & 3)));
        }
    }
}

template <typename T>
static void launch_norm(hipStream_t s, const norm_args& a)
{
    constexpr int E = 16 / sizeof(T);
    const int pieces = (a.cols + E - 1) / E;                 // of 16 bytes, one a thread and item
#define N(WAVES, ITEMS) hipLaunchKernelGGL((k_seq_norm<T, WAVES, ITEMS>), dim3(WAVES > 4 ? a.rows : (a.rows + 4 / WAVES - 1) / (4 / WAVES)), \
                                           dim3(WAVES > 4 ? WAVES * 64 : 256), 0, s, a)
    if (pieces <= 64) N(1, 1);
    else if (pieces <= 128) N(1, 2);
    else if (pieces <= 256) N(1, 4);
    else if (pieces <= 512) N(4, 2);
    else if (pieces <= 1024) N(4, 4);
    else if (pieces <= 2048) N(16, 2);
    else if (pieces <= 4096) N(16, 4);
    else N(16, 8);
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
