// Shared by the operators of include/rh_seq.h.
#pragma once
#include "rh_internal.h"
#include "rh_seq.h"

#define SEQ_E4M3_MAX 448.0f
#define SEQ_AMAX_MIN 0x1p-100f           // smaller largest magnitudes share a scale, so that its inverse stays finite

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;     // arrays of it stay in registers, where HIP's uint4 may not

__device__ __forceinline__ float seq_bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float seq_bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t seq_pack_bf16(float a, float b)
{
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
    const f32x2 v = {a, b};
    const bf16x2 r = __builtin_convertvector(v, bf16x2);     // round to nearest even
    return *(const uint32_t*)&r;
}
// two e4m3 values of a word (its low or high half) as two bf16, which hold them exactly
template <bool HIGH> __device__ __forceinline__ uint32_t seq_e4m3_pair(uint32_t u)
{
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HIGH);
    return *(const uint32_t*)&r;
}
// four floats to e4m3, rounded to nearest even (magnitudes up to 448 and a rounding error above)
__device__ __forceinline__ uint32_t seq_pack_e4m3(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// Four values over their scale, as e4m3.  Each quotient is rounded once, as a division's: the product with the reciprocal, corrected by its remainder (a fused
// multiplication leaves it exact), is that quotient wherever neither underflows; other scales are divided by.  (27600 tokens of 8 heads
// of 128 written in 44.9 us; divisions for all 52.7; products alone 43.7, which put what lies at a tie between two codes on either side.)
struct seq_scale { float value, inverse; };
__device__ __forceinline__ seq_scale seq_make_scale(float most) { const float v = most * (1.f / SEQ_E4M3_MAX); return {v, 1.f / v}; }
__device__ __forceinline__ uint32_t seq_pack_scaled(float a, float b, float c, float d, const seq_scale& s)
{
    if (!(s.value >= 0x1p-90f && s.value <= 0x1p120f)) return seq_pack_e4m3(a / s.value, b / s.value, c / s.value, d / s.value);
    auto over = [&](float v) { const float q = v * s.inverse; return fmaf(fmaf(-q, s.value, v), s.inverse, q); };
    return seq_pack_e4m3(over(a), over(b), over(c), over(d));
}

template <int N> struct seq_const { static constexpr int value = N; };

// Inclusive running sum over the wave's lanes, by row shifts and row broadcasts of the vector ALU.
__device__ __forceinline__ int32_t seq_scan(int32_t v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);        // the last lane of rows 0 and 2 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);        // lane 31 to the upper half
    return v;
}

__device__ __forceinline__ float seq_sum(float v)            // of the wave, the same for every lane
{
    auto from = [](float x, auto ctrl, auto rows) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, decltype(rows)::value, 0xF, decltype(rows)::value == 0xF));
    };
    v += from(v, seq_const<0x111>(), seq_const<0xF>());
    v += from(v, seq_const<0x112>(), seq_const<0xF>());
    v += from(v, seq_const<0x114>(), seq_const<0xF>());
    v += from(v, seq_const<0x118>(), seq_const<0xF>());
    v += from(v, seq_const<0x142>(), seq_const<0xA>());
    v += from(v, seq_const<0x143>(), seq_const<0xC>());
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// A vector in memory that need not be aligned: global loads and stores take any byte address, and one instruction
// that crosses a line costs less than one for every element.
template <typename V> struct __attribute__((packed, aligned(1))) seq_loose { V v; };
template <typename V> __device__ __forceinline__ V seq_load(const void* p) { return ((const seq_loose<V>*)p)->v; }
template <typename V> __device__ __forceinline__ void seq_store(void* p, V v) { ((seq_loose<V>*)p)->v = v; }

__device__ __forceinline__ float seq_to_f32(float v) { return v; }
__device__ __forceinline__ float seq_to_f32(__bf16 v) { return (float)v; }
__device__ __forceinline__ float seq_to_f32(uint8_t v) { return __builtin_amdgcn_cvt_f32_fp8((int)v, 0); }

// A whole division by a number that is fixed for the launch: floor(x / d) for 0 <= x < 2^31, by the high half of a product.
// With 2^s < d <= 2^(s+1) and m = ceil(2^(32+s) / d) < 2^32, x*m / 2^(32+s) passes x / d by less than x / 2^(32+s) < 2^-(s+1) <= 1 / d:
// the floor is right.  d = 1, whose m would not fit, goes by `one`, without a branch.
struct seq_div { uint32_t d, m, s, one; };
inline seq_div seq_make_div(uint32_t d)
{
    if (d <= 1) return {1, 0, 0, ~0u};
    const uint32_t s = 31 - (uint32_t)__builtin_clz(d - 1);  // 2^s <= d - 1 < 2^(s+1)
    return {d, (uint32_t)(((1ull << (32 + s)) + d - 1) / d), s, 0};
}
__device__ __forceinline__ uint32_t seq_quot(uint32_t x, const seq_div& v) { return (__umulhi(x, v.m) + (x & v.one)) >> v.s; }

// Scratch memory: rows of partial results of rh_cache_attend, or sums of slices of rh_matvec_packed, and as many counters as rows, which are zero between
// calls (rh_cache_plan takes the first).  A stream cut into n > 1 chunks has more than n - 1 >= n / 2 chunks' tiles, so that of ATTEND_CHUNKS chunks a CU twice as many at most
// belong to such streams.
#define ATTEND_CHUNKS 8          // chunks a CU of rh_cache_attend
#define SEQ_ROWS(ctx) (2 * ATTEND_CHUNKS * (ctx)->n_cu)
#define SEQ_ROW_BYTES(dim) (((dim) / 16 * 64 + 16) * 16)     // sums of 16 heads, and a maximum and a total of each
rh_status seq_counters(rh_ctx* ctx);
rh_status seq_scratch(rh_ctx* ctx);
// refusals of a cache; `name` is the call's
rh_status seq_check_cache(rh_ctx* ctx, const char* name, const rh_kv_cache* c);
