// rh_matvec_packed: products of a few rows with weights in 4 bits that share a scale by 32.
#include "seq_common.h"

struct matvec_args {
    const void* x;
    const float* x_scale;
    const uint8_t *w, *w_scale;
    void* y;
    int64_t x_stride, y_stride;
    int32_t rows, outs, ins, blocks, relu;
};

__device__ __forceinline__ float matvec_scale(uint8_t s)
{
    return s == 255 ? __builtin_nanf("") : __uint_as_float(s ? (uint32_t)s << 23 : 0x00400000u);     // 2^(s - 127), 2^-127 below the normal numbers
}
__device__ __forceinline__ float matvec_code(uint32_t c)
{
    const uint32_t m = c & 7;
    const float v = m < 2 ? 0.5f * (float)m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
    return c & 8 ? -v : v;
}

// One wave an output and row.
template <typename T, typename Y>
__global__ __launch_bounds__(256) void k_seq_matvec(matvec_args a)
{
    const int lane = threadIdx.x & 63, n = blockIdx.x * 4 + (threadIdx.x >> 6), m = blockIdx.y;
    if (n >= a.outs) return;
    const T* x = (const T*)a.x + m * a.x_stride;
    float sum = 0.f;
    for (int k = lane; k < a.ins; k += 64) {
        const uint8_t c = a.w[((int64_t)n * a.blocks + (k >> 5)) * 16 + ((k & 31) >> 1)];
        sum += seq_to_f32(x[k]) * (matvec_code(k & 1 ? c >> 4 : c & 15) * matvec_scale(a.w_scale[(int64_t)n * a.blocks + (k >> 5)]));
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane) return;
    if (a.x_scale) sum *= a.x_scale[m];
    if (a.relu) sum = sum < 0.f ? 0.f : sum;
    ((Y*)a.y)[m * a.y_stride + n] = (Y)sum;
}

template <typename T>
static void launch_matvec(hipStream_t s, const matvec_args& a, int y_type)
{
    const dim3 grid((a.outs + 3) / 4, a.rows);
    if (y_type == RH_T_F32) hipLaunchKernelGGL((k_seq_matvec<T, float>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_seq_matvec<T, __bf16>), grid, dim3(256), 0, s, a);
}

extern "C" rh_status rh_matvec_packed(rh_ctx* ctx, const void* x, int32_t x_type, int64_t x_stride, const float* x_scale,
                                      const uint8_t* w, const uint8_t* w_scale, int32_t n_rows, int32_t n_out, int32_t n_in,
                                      int32_t relu, void* y, int32_t y_type, int64_t y_stride)
{
    if (!ctx) return RH_E_INVALID;
    if (!w || !w_scale || (n_rows && (!x || !y))) RH_FAIL(ctx, RH_E_INVALID, "rh_matvec_packed: null argument");
    if (x_type != RH_T_F32 && x_type != RH_T_BF16 && x_type != RH_T_E4M3) RH_FAIL(ctx, RH_E_INVALID, "rh_matvec_packed: rows of type %d", x_type);
    if (y_type != RH_T_F32 && y_type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_matvec_packed: output of type %d", y_type);
    if (relu != 0 && relu != 1) RH_FAIL(ctx, RH_E_INVALID, "rh_matvec_packed: relu=%d", relu);
    if (n_rows < 0 || n_rows > 65535 || n_out < 1 || n_in < 1 || n_in > (1 << 20) || n_out > (1 << 26))
        RH_FAIL(ctx, RH_E_SHAPE, "rh_matvec_packed: %d rows, %d by %d weights", n_rows, n_out, n_in);
    if (x_stride < n_in || y_stride < n_out) RH_FAIL(ctx, RH_E_SHAPE, "rh_matvec_packed: a row stride below the row's length");
    if ((uintptr_t)w & 15) RH_FAIL(ctx, RH_E_INVALID, "rh_matvec_packed: w must be 16-byte aligned");
    if (n_rows == 0) return RH_OK;
    const matvec_args a = {x, x_scale, w, w_scale, y, x_stride, y_stride, n_rows, n_out, n_in, (n_in + 31) / 32, relu};
    if (x_type == RH_T_F32) launch_matvec<float>(ctx->stream, a, y_type);
    else if (x_type == RH_T_BF16) launch_matvec<__bf16>(ctx->stream, a, y_type);
    else launch_matvec<uint8_t>(ctx->stream, a, y_type);
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}
