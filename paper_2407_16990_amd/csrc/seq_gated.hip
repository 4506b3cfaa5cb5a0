// rh_norm_gated: x * SiLU(gate), root-mean-square norm over groups of its channels, and the norm's output in 8 bits.
//
// Bound by memory: x and the gate are read once, y and its 8-bit form written once.  A row belongs to one workgroup, a group of it to `lanes`
// neighbouring threads, with ITEMS pieces of 16 bytes a thread; pieces begin where groups do, at any address.  A row of more groups than the
// threads are for goes ROUNDS times around.  The products stay in registers between the sums of squares, the largest |y| of the row and the output.
// 27600 rows of 2048 in 8 groups of bf16, both outputs, inputs that no cache holds: 86 us, 4.6 TB/s; 14720 of 1540 in 4 groups of fp32 53, 5.1 TB/s; 8 of 2048, 8-bit output, 4.1.
// A group's lanes are rounded up to a power of two, a row's threads too: in groups that do not fill them many threads have nothing.  bf16, 8-bit output: 20000 rows of 3 groups of 264 52 us, of 256
// 22; 15000 of 16 of 72 36, of 64 18; 30000 of 520 28.5, of 512 19.5.  128 registers a thread are too few for fp32 groups of more than 16384 columns (19 spilled; 400 rows of 32768, both outputs,
// 49 us, 3.5 TB/s), and for 4 rounds of 4 pieces in fp32 (12), of 2 in bf16 (20) and 16 rounds (2).
// Several rows a workgroup, one after the other with the next one's loads ahead: 95 and 63 (two), 92 and 71 (four).
#include "seq_rows.h"
#include "seq_streams.h"

struct gated_args {
    const void *x, *gate;
    const float* weight;
    void* y;
    uint8_t* y8;
    float* y8_scale;
    int64_t x_stride, gate_stride;
    seq_div groups;
    int32_t rows, cols, per, lanes, log_lanes, rows_wg;      // per: channels a group; rows_wg: rows a workgroup
    float eps;
    bool past;
};

#define GATED_MAX_T 1024

// over `lanes` neighbouring threads, a power of two: lanes of a wave, or whole waves
template <bool MAX> __device__ __forceinline__ float gated_over(float v, int lanes, float* s_part)
{
    auto both = [](float a, float b) { return MAX ? (b != b || b > a ? b : a) : a + b; };
    for (int o = (lanes < 64 ? lanes : 64) / 2; o; o >>= 1) v = both(v, __shfl_xor(v, o));
    if (lanes > 64) {
        const int wave = threadIdx.x >> 6, n = lanes >> 6, first = wave / n * n;
        __syncthreads();                                     // what was there has been read
        if ((threadIdx.x & 63) == 0) s_part[wave] = v;
        __syncthreads();
        v = s_part[first];
        for (int w = 1; w < n; ++w) v = both(v, s_part[first + w]);
    }
    return v;
}

template <typename T, int ITEMS, int ROUNDS>
__global__ __launch_bounds__(GATED_MAX_T) void k_seq_gated(gated_args a)
{
    constexpr int E = 16 / sizeof(T);
    __shared__ float s_part[GATED_MAX_T / 64];
    __shared__ uint32_t s_most[GATED_MAX_T];
    const int t = threadIdx.x, lane = t & (a.lanes - 1);
    // a unit is a group of a row: of one row those of every round, or of several rows all of them
    const int unit = t >> a.log_lanes, sub = ROUNDS > 1 ? 0 : (int)seq_quot((uint32_t)unit, a.groups), units = (int)blockDim.x >> a.log_lanes;
    const int64_t row = (int64_t)blockIdx.x * a.rows_wg + sub;
    const bool here = sub < a.rows_wg && row < a.rows;
    const T *x = (const T*)a.x + (here ? row : 0) * a.x_stride, *z = (const T*)a.gate + (here ? row : 0) * a.gate_stride;
    if (a.y8) {
        if (t < a.rows_wg) s_most[t] = 0;
    }
    constexpr int AHEAD = ROUNDS * ITEMS <= 4 ? ROUNDS : ITEMS < 4 ? 4 / ITEMS : 1;      // rounds whose loads are in flight together
    // weights on their way before the sums: 14720 rows of 1540 in 4 groups, fp32, 59.2 -> 53.1 us; not in bf16, whose two loads for a piece of x come in between (27600 of 2048 in 8, both outputs, 90 -> 97)
    constexpr bool EARLY = sizeof(T) == 4 && ROUNDS * ITEMS <= 2;
    u32x4 wr[EARLY ? ROUNDS : 1][ITEMS][E / 4];
    float v[ROUNDS][ITEMS][E], most = 0.f;
    u32x4 in[AHEAD][ITEMS], open[AHEAD][ITEMS];
    auto group = [&](int round) { return ROUNDS > 1 ? unit + round * units : unit - sub * (int)a.groups.d; };
    auto live = [&](int round) { return here && group(round) < (int)a.groups.d; };
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if (r % AHEAD == 0) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const int first = live(r + k) ? group(r + k) * a.per : 0;
                    in[k][i] = row_load<T, E>(x + first, (lane + i * a.lanes) * E, a.per);
                    open[k][i] = row_load<T, E>(z + first, (lane + i * a.lanes) * E, a.per);
                }
        }
        const int first = live(r) ? group(r) * a.per : 0;
        auto weights = [&](u32x4 (&to)[ITEMS][E / 4]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < E; e += 4) to[i][e / 4] = row_load<float, 4>(a.weight + first, (lane + i * a.lanes) * E + e, a.per);
        };
        if (EARLY) weights(wr[r]);
        float square = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float g[E];
            row_place<T, E>(in[r % AHEAD][i], (lane + i * a.lanes) * E, a.per, v[r][i]);
            row_place<T, E>(open[r % AHEAD][i], (lane + i * a.lanes) * E, a.per, g);
#pragma unroll
            for (int e = 0; e < E; ++e) { v[r][i][e] *= seq_silu(g[e]); square = fmaf(v[r][i][e], v[r][i][e], square); }
        }
        square = gated_over<false>(square, a.lanes, s_part);
        const float scale = 1.f / sqrtf(square / (float)a.per + a.eps);
        if (!EARLY) weights(wr[0]);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (lane + i * a.lanes) * E, n = a.per - c;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                float w[4];
                row_place<float, 4>(wr[EARLY ? r : 0][i][e / 4], c + e, a.per, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[r][i][e + k] = v[r][i][e + k] * scale * w[k];
                    const float m = fabsf(v[r][i][e + k]);
                    if (live(r)) most = m != m || m > most ? m : most;
                }
            }
            if (a.y && live(r) && n > 0) row_store<T, E>((T*)a.y + row * a.cols + first + c, n, v[r][i], a.past);
        }
    }
    if (!a.y8) return;
    // the largest of the row: magnitudes compare as whole numbers, a NaN above all
    most = gated_over<true>(most, a.lanes < 64 ? a.lanes : 64, nullptr);
    __syncthreads();
    if (here && (t & ((a.lanes < 64 ? a.lanes : 64) - 1)) == 0) atomicMax(&s_most[sub], __float_as_uint(most) & 0x7FFFFFFFu);
    __syncthreads();
    if (!here) return;
    most = __uint_as_float(s_most[sub]);
    most = most < SEQ_AMAX_MIN ? SEQ_AMAX_MIN : most;
    const seq_scale y8_scale = seq_make_scale(most);
    if (lane == 0 && unit == sub * (ROUNDS > 1 ? 0 : (int)a.groups.d)) a.y8_scale[row] = y8_scale.value;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if (!live(r)) continue;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (lane + i * a.lanes) * E, n = a.per - c;
            if (n <= 0) continue;
            uint8_t* o = a.y8 + row * a.cols + group(r) * a.per + c;
            u32x4 q = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < E; e += 4) q[e / 4] = seq_pack_scaled(v[r][i][e], v[r][i][e + 1], v[r][i][e + 2], v[r][i][e + 3], y8_scale);
            if (n < E) row_put<1>(o, n, q);
            else if constexpr (E == 8) { const uint64_t w = (uint64_t)q[1] << 32 | q[0]; if (a.past) seq_store_past(o, w); else seq_store(o, w); }
            else { if (a.past) seq_store_past(o, (uint32_t)q[0]); else seq_store(o, (uint32_t)q[0]); }
        }
    }
}

template <typename T>
static bool launch_gated(hipStream_t s, gated_args& a)       // false: more workgroups than a launch takes
{
    constexpr int E = 16 / sizeof(T);
    const int pieces = (a.per + E - 1) / E;
    int items = 1;
    a.log_lanes = 0;
    while (a.log_lanes < 10 && pieces > (1 << a.log_lanes) * (a.log_lanes < 6 ? 1 : 2)) ++a.log_lanes;
    a.lanes = 1 << a.log_lanes;
    while (items * a.lanes < pieces) items *= 2;
    const int64_t wide = (int64_t)a.groups.d * a.lanes;      // threads of a row
    int rounds = 1, threads = 256;
    while (wide > (int64_t)rounds * GATED_MAX_T) rounds *= 2;
    if (rounds > 1) threads = GATED_MAX_T;
    else while (threads < wide) threads *= 2;
    a.rows_wg = rounds > 1 ? 1 : (int)(threads / wide);
    const int64_t wgs = ((int64_t)a.rows + a.rows_wg - 1) / a.rows_wg;
    if (wgs * threads > 0xFFFFFFFFll) return false;
    const dim3 grid((unsigned)wgs);
#define N(ITEMS, ROUNDS) hipLaunchKernelGGL((k_seq_gated<T, ITEMS, ROUNDS>), grid, dim3(threads), 0, s, a)
    // a row has 4096 pieces (bf16) or 8192 (fp32) at most, and more than half of a group's places for them are taken
    if (rounds == 1) { if (items == 1) N(1, 1); else if (items == 2) N(2, 1); else if (items == 4) N(4, 1); else if constexpr (E == 4) N(8, 1); }
    else if (rounds == 2) { if (items == 1) N(1, 2); else if (items == 2) N(2, 2); else if constexpr (E == 4) N(4, 2); }
    else if (rounds == 4) { if (items == 1) N(1, 4); else if (items == 2) N(2, 4); else if constexpr (E == 4) N(4, 4); }
    else if (rounds == 8) { if (items == 1) N(1, 8); else if constexpr (E == 4) N(2, 8); }
    else if constexpr (E == 4) N(1, 16);
#undef N
    return true;
}

extern "C" rh_status rh_norm_gated(rh_ctx* ctx, const void* x, int64_t x_stride, const void* gate, int64_t gate_stride, const float* weight,
                                   int32_t type, int32_t n_rows, int32_t n_cols, int32_t groups, float eps, void* y, uint8_t* y8,
                                   float* y8_scale)
{
    if (!ctx) return RH_E_INVALID;
    if (!weight || (n_rows && (!x || !gate))) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_gated: null argument");
    if (n_rows && !y8 != !y8_scale) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_gated: 8-bit output and its scales go together");
    if (n_rows && !y && !y8) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_gated: no output asked for");
    if (type != RH_T_F32 && type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_gated: rows of type %d", type);
    if (n_rows < 0 || n_cols < 1 || n_cols > RH_SEQ_MAX_COLS)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_norm_gated: %d rows of %d elements (1 to %d)", n_rows, n_cols, RH_SEQ_MAX_COLS);
    if (groups < 1 || groups > RH_SEQ_MAX_GROUPS || n_cols % groups)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_norm_gated: %d elements in %d groups (1 to %d)", n_cols, groups, RH_SEQ_MAX_GROUPS);
    if (x_stride < n_cols || gate_stride < n_cols) RH_FAIL(ctx, RH_E_SHAPE, "rh_norm_gated: a row stride below %d", n_cols);
    if (!(eps >= 0.f)) RH_FAIL(ctx, RH_E_INVALID, "rh_norm_gated: eps must not be negative");
    if (n_rows == 0) return RH_OK;
    gated_args a;
    a.x = x; a.gate = gate; a.weight = weight; a.y = y; a.y8 = y8; a.y8_scale = y8_scale; a.x_stride = x_stride; a.gate_stride = gate_stride;
    a.groups = seq_make_div((uint32_t)groups); a.rows = n_rows; a.cols = n_cols; a.per = n_cols / groups; a.eps = eps;
    a.past = (int64_t)n_rows * n_cols * (type == RH_T_F32 ? 4 : 2) >= ROWS_PAST;
    if (!(type == RH_T_F32 ? launch_gated<float>(ctx->stream, a) : launch_gated<__bf16>(ctx->stream, a)))
        RH_FAIL(ctx, RH_E_SHAPE, "rh_norm_gated: %d rows of %d elements", n_rows, n_cols);
    RH_HIP(ctx, hipGetLastError());
    return RH_OK;
}
