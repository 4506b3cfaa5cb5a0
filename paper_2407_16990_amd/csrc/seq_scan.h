// rh_state_scan: a selective scan of every stream's state over its tokens.  Both types' sources include this.
//
// A lane has four of the up to 128 states of a channel, so that LN = 1, 2, 4 ... 32 lanes have a channel's; what they add to y is summed over them by exchanges inside the wave.
// Single tokens: the states, 2 * 4 * n bytes a channel, are all that counts; a lane loads and stores 16 bytes of them.
// Many tokens: bound by the vector instructions of h = exp2(delta a) h + delta x b, y += c h: a power of two takes as long as four others.  A
// workgroup has CH channels of a stream and goes through its rows, SCAN_ROWS of them staged in LDS at a time: delta and delta * x of every
// channel, worked out once, b and c in fp32; the next rows' loads are in flight meanwhile.  y takes delta's place.
#pragma once
#include "seq_rows.h"
#include "seq_streams.h"

#define SCAN_ROOM(ctx) ((int64_t)SEQ_ROWS(ctx) * SEQ_ROW_BYTES(RH_SEQ_MAX_DIM) / (int64_t)sizeof(float))     // floats of the scratch memory

struct scan_args {
    streams_args r;
    const void *x, *dt, *gate, *b, *c;
    const float *a, *dt_bias, *skip;
    float *state, *ws;           // ws: of chunk rows, the states [row][channels][4 * LN], then the sums of delta [row][channels]
    void* y;
    int64_t x_stride, dt_stride, gate_stride, b_stride, c_stride, y_stride;
    seq_div per, blocks, group_blocks;       // channels a group; workgroups' channel blocks, in all and of a group
    int32_t channels, n, softplus, chunk, ws_rows;
};

// exp(v), off by an ulp or two: the rounding of v * log2(e) is made up for behind the power of two
__device__ __forceinline__ float scan_exp(float v)
{
    const float hi = v * 1.44269504089f, lo = fmaf(v, 1.44269504089f, -hi) + v * 1.92596299e-8f;
    const float e = __builtin_amdgcn_exp2f(hi);
    return fmaf(e, lo * 0.69314718056f, e);
}
// log(1 + exp(v)): with w = 1 + e rounded, log(w) * e / (w - 1) makes up for the rounding (Goldberg 1991, theorem 4); above 20 it is v to half an ulp
__device__ __forceinline__ float scan_softplus(float v)
{
    const float e = scan_exp(v), w = 1.f + e, d = w - 1.f;
    const float l = __builtin_amdgcn_logf(w) * 0.69314718056f;
    const float s = d == 0.f ? e : l * (e * __builtin_amdgcn_rcpf(d));
    return v > 20.f ? v : s;
}

// the sum over LN neighbouring lanes, the same for all of them
template <int LN> __device__ __forceinline__ float scan_over(float v)
{
    auto with = [](float x, auto ctrl) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    if constexpr (LN >= 2) v += with(v, seq_const<0xB1>());  // lane ^ 1
    if constexpr (LN >= 4) v += with(v, seq_const<0x4E>());  // lane ^ 2
    if constexpr (LN >= 8) v += with(v, seq_const<0x141>()); // mirrored in 8
    if constexpr (LN >= 16) v += with(v, seq_const<0x140>());        // in 16
    if constexpr (LN >= 32) v += __shfl_xor(v, 16);
    return v;
}

// four elements from i on, of n; zeros behind
template <typename T, bool FULL> __device__ __forceinline__ f32x4 scan_quad(const T* p, int i, int n)
{
    if constexpr (FULL) {
        if constexpr (sizeof(T) == 4) return seq_load<f32x4>(p + i);
        else {
            const uint2 u = seq_load<uint2>(p + i);
            return f32x4{seq_bf16_lo(u.x), seq_bf16_hi(u.x), seq_bf16_lo(u.y), seq_bf16_hi(u.y)};
        }
    } else {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = i + e < n ? seq_to_f32(p[i + e]) : 0.f;
        return v;
    }
}
template <bool FULL> __device__ __forceinline__ void scan_put(float* p, int i, int n, f32x4 v)
{
    if constexpr (FULL) seq_store(p + i, v);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e) if (i + e < n) p[i + e] = v[e];
}

// ---------------------------------------------------------------------------------------------------------------
// one row a stream
// ---------------------------------------------------------------------------------------------------------------
// FULL: n = 4 * LN.  R streams a thread, whose loads are in flight together.
template <typename T, int LN, bool FULL, int R>
__global__ __launch_bounds__(256) void k_seq_scan_step(scan_args a)
{
    const int j = threadIdx.x % LN;
    const uint32_t blk = blockIdx.x, part = seq_quot(blk, a.blocks);
    const int c0 = (int)(blk - part * a.blocks.d) * (256 / LN) + threadIdx.x / LN, c = c0 < a.channels ? c0 : a.channels - 1;
    const int g = (int)seq_quot((uint32_t)c, a.per);
    f32x4 h[R], b[R], cc[R];
    float x[R], dt[R], gate[R];
    int32_t to[R];
    const int64_t at = (int64_t)c * a.n, pool = (int64_t)a.channels * a.n;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t s = (int64_t)part * R + i < a.r.n_rows ? (int64_t)part * R + i : a.r.n_rows - 1;
        const int32_t from = streams_slot(a.r, (int)s);
        to[i] = streams_into(a.r, (int)s);
        h[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (from >= 0) h[i] = scan_quad<float, FULL>(a.state + from * pool + at, 4 * j, a.n);
        b[i] = scan_quad<T, FULL>((const T*)a.b + s * a.b_stride + (int64_t)g * a.n, 4 * j, a.n);
        cc[i] = scan_quad<T, FULL>((const T*)a.c + s * a.c_stride + (int64_t)g * a.n, 4 * j, a.n);
        x[i] = seq_to_f32(((const T*)a.x)[s * a.x_stride + c]);
        dt[i] = seq_to_f32(((const T*)a.dt)[s * a.dt_stride + c]);
        gate[i] = a.gate ? seq_to_f32(((const T*)a.gate)[s * a.gate_stride + c]) : 0.f;
    }
    const f32x4 fade = scan_quad<float, FULL>(a.a + at, 4 * j, a.n) * 1.44269504089f;
    const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, skip = a.skip ? a.skip[c] : 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float d = dt[i] + bias;
        d = a.softplus ? scan_softplus(d) : d;
        const float u = d * x[i];
        float y = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[i][e] = fmaf(__builtin_amdgcn_exp2f(d * fade[e]), h[i][e], u * b[i][e]);
            if (FULL || 4 * j + e < a.n) y = fmaf(cc[i][e], h[i][e], y);
        }
        y = scan_over<LN>(y);
        const int64_t s = (int64_t)part * R + i;
        if (c0 >= a.channels || s >= a.r.n_rows) continue;
        if (to[i] >= 0) scan_put<FULL>(a.state + to[i] * pool + at, 4 * j, a.n, h[i]);
        if (j) continue;
        if (a.skip) y = fmaf(skip, x[i], y);
        if (a.gate) y *= seq_silu(gate[i]);
        ((T*)a.y)[s * a.y_stride + c] = (T)y;
    }
}

// ---------------------------------------------------------------------------------------------------------------
// many rows a stream
// ---------------------------------------------------------------------------------------------------------------
// A stream of `len` rows is cut into chunks of equal length, a.chunk rows or so; below one and a half it stays whole.
template <int ROWS> struct scan_cut {
    int32_t size, n;
    __device__ __forceinline__ scan_cut(int32_t len, int32_t chunk)
    {
        n = (int32_t)(((uint32_t)len + (uint32_t)chunk / 2) / (uint32_t)chunk);
        if (n < 2) { size = len; n = len > 0; return; }
        size = (int32_t)(((uint32_t)len + n - 1) / (uint32_t)n + ROWS - 1) / ROWS * ROWS;
        n = (int32_t)(((uint32_t)len + size - 1) / (uint32_t)size);                         // rounded up to whole stages, fewer may do
    }
};
// what a workgroup counts of a stream to find its own: its chunks, those that leave something to the next, or the streams that are cut
enum { SCAN_ALL, SCAN_SUMS, SCAN_CARRY };

// The stream that the workgroup's index q falls in, its place in it, and the row of ws where the stream's chunks begin; false where there is none.
template <int ROWS, int WHAT>
__device__ __forceinline__ bool scan_find(const scan_args& a, int32_t q, int32_t* s_mem, int32_t* s_wave, int& b, int32_t& place, int32_t& row)
{
    auto own = [&](int32_t len) { const scan_cut<ROWS> k(len, a.chunk); return WHAT == SCAN_ALL ? k.n : k.n < 2 ? 0 : WHAT == SCAN_SUMS ? k.n - 1 : 1; };
    auto rows = [&](int32_t len) { const scan_cut<ROWS> k(len, a.chunk); return k.n < 2 ? 0 : k.n; };
    if (a.r.n_streams <= 64) {                               // a stream a lane
        const int lane = threadIdx.x & 63;
        int32_t begin = 0, end = 0;
        if (lane < a.r.n_streams) streams_rows(a.r, lane, begin, end);
        const int32_t mine = own(end - begin), wide = rows(end - begin), upto = seq_scan(mine), ahead = seq_scan(wide) - wide;
        const uint64_t hit = __ballot(q >= upto - mine && q < upto);
        if (!hit) return false;
        b = __builtin_ctzll(hit);
        place = q - __builtin_amdgcn_readlane(upto - mine, b);
        row = __builtin_amdgcn_readlane(ahead, b);
    } else {
        int32_t* s_rows = s_mem + a.r.n_streams + 1;
        streams_sums(a.r, s_mem, s_wave, own);
        streams_sums(a.r, s_rows, s_wave, rows);
        if (q >= s_mem[a.r.n_streams]) return false;
        b = __builtin_amdgcn_readfirstlane(streams_find(s_mem, a.r.n_streams, q));
        place = q - __builtin_amdgcn_readfirstlane(s_mem[b]);
        row = __builtin_amdgcn_readfirstlane(s_rows[b]);
    }
    return place >= 0;
}

template <typename T, int LN, int K> struct scan_shape {
    static constexpr int E = 16 / sizeof(T), CH = 256 / LN * K;
    static constexpr int BY_X = 4096 / CH, BY_B = 1024 / LN, MOST = 64;
    static constexpr int ROWS = (BY_X < BY_B ? BY_X : BY_B) < MOST ? (BY_X < BY_B ? BY_X : BY_B) : MOST;     // 32 KB of LDS for delta and delta * x, or for b and c, at most
    static constexpr int PIECES = ROWS * CH / E, NX = (PIECES + 255) / 256;              // of 16 bytes of x, a stage's and a thread's
    static constexpr int QUADS = ROWS * LN, NB = (QUADS + 255) / 256;                    // of b, and of c
    static constexpr int LDS = ROWS * (CH * 2 + LN * 8) * 4;
};

// OUT: y and the states behind the streams' last rows.  Otherwise what a chunk makes of a state of zeros, and the sum of its delta, for the next one.
template <typename T, int LN, int K, bool FULL, bool OUT>
__global__ __launch_bounds__(256) void k_seq_scan(scan_args a)
{
    typedef scan_shape<T, LN, K> S;
    constexpr int E = S::E, CH = S::CH, ROWS = S::ROWS, NX = S::NX, NB = S::NB, LW = LN < 4 ? LN : 4;
    extern __shared__ f32x4 s_stage[];
    __shared__ int32_t s_wave[STREAMS_T / 64];
    float* s_du = (float*)s_stage;                           // [row][channel]: delta and delta * x, then y
    f32x4 *s_b = (f32x4*)(s_du + ROWS * CH * 2), *s_c = s_b + ROWS * LN;

    const int t = threadIdx.x, j = t % LN, cl = t / LN * K;
    const uint32_t item = seq_quot(blockIdx.x, a.blocks), blk = blockIdx.x - item * a.blocks.d;
    int b;
    int32_t place, ws_row;
    if (!scan_find<ROWS, OUT ? SCAN_ALL : SCAN_SUMS>(a, (int32_t)item, (int32_t*)s_stage, s_wave, b, place, ws_row)) return;
    int32_t begin, end;
    streams_rows(a.r, b, begin, end);
    const scan_cut<ROWS> cut(end - begin, a.chunk);
    if (place >= cut.n || (cut.n > 1 && ws_row + cut.n > a.ws_rows)) return;                // offsets that do not ascend
    const int32_t first = begin + place * cut.size, stop = end - first < cut.size ? end : first + cut.size;
    const int g = (int)seq_quot(blk, a.group_blocks);
    const int c_end = (g + 1) * (int)a.per.d, c_blk = g * (int)a.per.d + (int)(blk - (uint32_t)g * a.group_blocks.d) * CH;       // the group's last channel + 1, this block's first
    const int64_t pool = (int64_t)a.channels * a.n;
    float* sums = a.ws + (int64_t)a.ws_rows * a.channels * (4 * LN);

    // ---- this lane's states
    f32x4 h[K], fade[K];
    float total[K];
    {
        const int32_t from = cut.n < 2 ? streams_slot(a.r, b) : -1;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = c_blk + cl + k < c_end ? c_blk + cl + k : c_end - 1;
            fade[k] = scan_quad<float, FULL>(a.a + (int64_t)c * a.n, 4 * j, a.n) * 1.44269504089f;
            h[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            total[k] = 0.f;
            if (OUT && cut.n > 1) h[k] = *(const f32x4*)(a.ws + ((int64_t)(ws_row + place) * a.channels + c) * (4 * LN) + 4 * j);
            else if (OUT && from >= 0) h[k] = scan_quad<float, FULL>(a.state + from * pool + (int64_t)c * a.n, 4 * j, a.n);
        }
    }

    // ---- this thread's pieces of the rows: E channels, the same of every row that it has
    constexpr int PR = CH / E;                               // pieces a row
    const int pc = t % PR * E, pr = t / PR, cg = c_blk + pc, left = c_end - cg;
    float bias[E], skip[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        bias[e] = a.dt_bias && e < left ? a.dt_bias[cg + e] : 0.f;
        skip[e] = OUT && a.skip && e < left ? a.skip[cg + e] : 0.f;
    }
    struct raw { u32x4 x[NX], dt[NX]; f32x4 b[NB], c[NB]; };
    u32x4 gate[NX];
    auto load = [&](int32_t row, raw& in) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int r = i * (256 / PR) + pr;
            const int64_t at = row + r < stop ? row + r : stop - 1;
            if (S::PIECES < 256 && r >= ROWS) { in.x[i] = in.dt[i] = u32x4{0, 0, 0, 0}; continue; }
            in.x[i] = row_load<T, E>((const T*)a.x + at * a.x_stride, cg, c_end);
            in.dt[i] = row_load<T, E>((const T*)a.dt + at * a.dt_stride, cg, c_end);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int q = i * 256 + t, r = q / LN;
            const int64_t at = row + r < stop ? row + r : stop - 1;
            in.b[i] = scan_quad<T, FULL>((const T*)a.b + at * a.b_stride + (int64_t)g * a.n, 4 * (q % LN), a.n);
            if (OUT) in.c[i] = scan_quad<T, FULL>((const T*)a.c + at * a.c_stride + (int64_t)g * a.n, 4 * (q % LN), a.n);
        }
    };
    raw in;
    load(first, in);
    if (a.r.n_streams > 64) __syncthreads();                 // the counts there have been read
    for (int32_t row = first; row < stop; row += ROWS) {
        const int rows = stop - row < ROWS ? stop - row : ROWS;
        // ---- into LDS; rows behind the last leave the state as it is: delta, delta * x and b are zero
        float x[NX][E];
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int r = i * (256 / PR) + pr;
            float dt[E];
            row_place<T, E>(in.x[i], cg, c_end, x[i]);
            row_place<T, E>(in.dt[i], cg, c_end, dt);
            if (S::PIECES < 256 && r >= ROWS) continue;
            float* to = s_du + (r * CH + pc) * 2;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                f32x4 v;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float d = dt[e + k] + bias[e + k];
                    d = a.softplus ? scan_softplus(d) : d;
                    v[2 * k] = r < rows ? d : 0.f;
                    v[2 * k + 1] = r < rows ? d * x[i][e + k] : 0.f;
                }
                *(f32x4*)(to + 2 * e) = v;
            }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int q = i * 256 + t, r = q / LN;
            if (S::QUADS % 256 && q >= S::QUADS) continue;
            s_b[q] = r < rows ? in.b[i] : f32x4{0.f, 0.f, 0.f, 0.f};
            if (OUT) s_c[q] = in.c[i];
        }
        __syncthreads();
        // ---- the next rows' loads, and these rows' gate
        if (OUT && a.gate) {
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                const int r = i * (256 / PR) + pr;
                if (S::PIECES < 256 && r >= ROWS) continue;
                const int64_t at = row + r < stop ? row + r : stop - 1;
                gate[i] = row_load<T, E>((const T*)a.gate + at * a.gate_stride, cg, c_end);
            }
        }
        if (row + ROWS < stop) load(row + ROWS, in);
        // ---- the rows
        for (int r0 = 0; r0 < rows; r0 += 4) {
            float mine[K][4 / LW];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i;
                const f32x4 bq = s_b[r * LN + j], cq = OUT ? s_c[r * LN + j] : f32x4{0.f, 0.f, 0.f, 0.f};
                float du[2 * K];
#pragma unroll
                for (int k = 0; k < 2 * K; k += 2) {
                    if constexpr (K % 2 == 0) {
                        if (k % 4 == 0) { const f32x4 v = *(const f32x4*)(s_du + (r * CH + cl) * 2 + k); du[k] = v[0]; du[k + 1] = v[1]; du[k + 2] = v[2]; du[k + 3] = v[3]; }
                    } else { const float2 v = *(const float2*)(s_du + (r * CH + cl) * 2 + k); du[k] = v.x; du[k + 1] = v.y; }
                }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float y = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        h[k][e] = fmaf(__builtin_amdgcn_exp2f(du[2 * k] * fade[k][e]), h[k][e], du[2 * k + 1] * bq[e]);
                        if (!FULL && 4 * j + e >= a.n) h[k][e] = 0.f;       // an infinite delta * x times the zero there
                        if (OUT) y = e ? fmaf(cq[e], h[k][e], y) : cq[e] * h[k][e];
                    }
                    if constexpr (OUT) {
                        y = scan_over<LN>(y);
                        mine[k][i / LW] = i % LW == 0 || i % LW == j % LW ? y : mine[k][i / LW];
                    } else total[k] += du[2 * k];
                }
            }
            if (OUT && j < LW) {
#pragma unroll
                for (int i = 0; i < 4 / LW; ++i)
#pragma unroll
                    for (int k = 0; k < K; ++k) s_du[((r0 + i * LW + j % LW) * CH + cl + k) * 2] = mine[k][i];
            }
        }
        __syncthreads();
        // ---- y: the thread's own pieces, which it also fills with the next rows
        if constexpr (OUT) {
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                const int r = i * (256 / PR) + pr;
                if (r >= rows) continue;
                float y[E], z[E];
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const f32x4 v = *(const f32x4*)(s_du + (r * CH + pc + e) * 2);
                    y[e] = v[0]; y[e + 1] = v[2];
                }
                if (a.skip)
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] = fmaf(skip[e], x[i][e], y[e]);
                if (a.gate) {
                    row_place<T, E>(gate[i], cg, c_end, z);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] *= seq_silu(z[e]);
                }
                if (left > 0) row_store<T, E>((T*)a.y + (int64_t)(row + r) * a.y_stride + cg, left, y);
            }
        }
    }
    // ---- the state behind the last row
    const int32_t to = OUT && place == cut.n - 1 ? streams_into(a.r, b) : -1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = c_blk + cl + k;
        if (c >= c_end) continue;
        if (!OUT) {
            const int64_t at = (int64_t)(ws_row + place) * a.channels + c;
            *(f32x4*)(a.ws + at * (4 * LN) + 4 * j) = h[k];
            if (j == 0) sums[at] = total[k];
        } else if (to >= 0) scan_put<FULL>(a.state + to * pool + (int64_t)c * a.n, 4 * j, a.n, h[k]);
    }
}

// The states that the chunks of the cut streams begin with, in the place of what each makes of zeros: h = exp(a * sum of delta) h + that, chunk after chunk.
#define SCAN_AHEAD 8             // chunks whose loads are in flight
template <int LN, int ROWS, bool FULL>
__global__ __launch_bounds__(256) void k_seq_scan_carry(scan_args a)
{
    extern __shared__ f32x4 s_stage[];
    __shared__ int32_t s_wave[STREAMS_T / 64];
    int b;
    int32_t place, ws_row;
    const uint32_t item = seq_quot(blockIdx.x, a.blocks);
    if (!scan_find<ROWS, SCAN_CARRY>(a, (int32_t)item, (int32_t*)s_stage, s_wave, b, place, ws_row)) return;
    int32_t begin, end;
    streams_rows(a.r, b, begin, end);
    const scan_cut<ROWS> cut(end - begin, a.chunk);
    if (place > 0 || cut.n < 2 || ws_row + cut.n > a.ws_rows) return;
    const int c = (int)(blockIdx.x - item * a.blocks.d) * (256 / LN) + threadIdx.x / LN, j = threadIdx.x % LN;
    if (c >= a.channels) return;
    const int32_t from = streams_slot(a.r, b);
    const f32x4 fade = scan_quad<float, FULL>(a.a + (int64_t)c * a.n, 4 * j, a.n) * 1.44269504089f;
    f32x4 h = {0.f, 0.f, 0.f, 0.f};
    if (from >= 0) h = scan_quad<float, FULL>(a.state + (int64_t)from * a.channels * a.n + (int64_t)c * a.n, 4 * j, a.n);
    const int64_t step = (int64_t)a.channels * (4 * LN);
    float* at = a.ws + ((int64_t)ws_row * a.channels + c) * (4 * LN) + 4 * j;
    const float* sum = a.ws + (int64_t)a.ws_rows * step + (int64_t)ws_row * a.channels + c;
    for (int32_t k0 = 0; k0 < cut.n; k0 += SCAN_AHEAD) {
        f32x4 add[SCAN_AHEAD];
        float total[SCAN_AHEAD];
#pragma unroll
        for (int i = 0; i < SCAN_AHEAD; ++i) {
            const int32_t k = k0 + i < cut.n - 1 ? k0 + i : 0;               // the last chunk leaves nothing
            add[i] = *(const f32x4*)(at + k * step);
            total[i] = sum[(int64_t)k * a.channels];
        }
#pragma unroll
        for (int i = 0; i < SCAN_AHEAD; ++i) {
            if (k0 + i >= cut.n) break;
            *(f32x4*)(at + (k0 + i) * step) = h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = fmaf(__builtin_amdgcn_exp2f(total[i] * fade[e]), h[e], add[i][e]);
        }
    }
}

template <typename T, int LN, bool FULL>
static hipError_t launch_scan(rh_ctx* ctx, scan_args& a, rh_status* failed)
{
    constexpr int K = 2;
    typedef scan_shape<T, LN, K> S;
    const int groups = a.channels / (int)a.per.d;
    const int64_t wide = (a.channels + 256 / LN - 1) / (256 / LN);           // workgroups of one channel a thread
    if (!a.r.offsets) {
        a.blocks = seq_make_div((uint32_t)wide);
        if (wide * a.r.n_rows >= 16 * (int64_t)ctx->n_cu) hipLaunchKernelGGL((k_seq_scan_step<T, LN, FULL, 4>), dim3((unsigned)(((int64_t)a.r.n_rows + 3) / 4 * wide)), dim3(256), 0, ctx->stream, a);
        else hipLaunchKernelGGL((k_seq_scan_step<T, LN, FULL, 1>), dim3((unsigned)(a.r.n_rows * wide)), dim3(256), 0, ctx->stream, a);
        return hipGetLastError();
    }
    const int group_blocks = ((int)a.per.d + S::CH - 1) / S::CH;
    const int64_t blocks = (int64_t)groups * group_blocks;
    // rows a chunk: enough workgroups for the GPU where streams are few, and no more states than the scratch memory holds
    const int64_t room = SCAN_ROOM(ctx) / ((int64_t)a.channels * (4 * LN + 1));
    const int64_t least = room > 0 ? (int64_t)a.r.n_rows * 4 / (3 * room) + 1 : 0x3FFFFFFF;
    int64_t chunk = (int64_t)a.r.n_rows * blocks / (2 * ctx->n_cu);
    chunk = chunk < 4 * S::ROWS ? 4 * S::ROWS : chunk;
    chunk = chunk < 128 ? 128 : chunk;
    chunk = chunk < least ? least : chunk;
    a.chunk = (int32_t)(chunk > 0x3FFFFFFF ? 0x3FFFFFFF : chunk);
    const bool cut = 2 * (int64_t)a.r.n_rows >= 3 * (int64_t)a.chunk;        // otherwise no stream can be as long
    a.ws_rows = cut ? (int32_t)((int64_t)a.r.n_rows * 4 / (3 * (int64_t)a.chunk)) + 1 : 0;
    const size_t counts = a.r.n_streams > 64 ? 2 * (a.r.n_streams + 1) * sizeof(int32_t) : 0;
    const size_t lds = S::LDS > counts ? S::LDS : counts;
    if (cut) {
        const rh_status st = seq_scratch(ctx);
        if (st != RH_OK) { *failed = st; return hipSuccess; }
        a.ws = (float*)ctx->seq_ws;
        a.blocks = seq_make_div((uint32_t)blocks);
        a.group_blocks = seq_make_div((uint32_t)group_blocks);
        hipLaunchKernelGGL((k_seq_scan<T, LN, K, FULL, false>), dim3((unsigned)(((int64_t)a.r.n_rows / a.chunk + 1) * blocks)), dim3(256), lds, ctx->stream, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.blocks = seq_make_div((uint32_t)wide);
        const int64_t most = (int64_t)a.r.n_rows * 2 / (3 * (int64_t)a.chunk) + 1;       // streams that are cut
        hipLaunchKernelGGL((k_seq_scan_carry<LN, S::ROWS, FULL>), dim3((unsigned)((most < a.r.n_streams ? most : a.r.n_streams) * wide)), dim3(256), counts, ctx->stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    a.blocks = seq_make_div((uint32_t)blocks);
    a.group_blocks = seq_make_div((uint32_t)group_blocks);
    hipLaunchKernelGGL((k_seq_scan<T, LN, K, FULL, true>), dim3((unsigned)(((int64_t)a.r.n_rows / a.chunk + a.r.n_streams) * blocks)), dim3(256), lds, ctx->stream, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_scan(rh_ctx* ctx, scan_args& a, rh_status* failed)
{
#define N(LN) return a.n == 4 * LN ? launch_scan<T, LN, true>(ctx, a, failed) : launch_scan<T, LN, false>(ctx, a, failed)
    if (a.n <= 4) N(1);
    if (a.n <= 8) N(2);
    if (a.n <= 16) N(4);
    if (a.n <= 32) N(8);
    if (a.n <= 64) N(16);
    N(32);
#undef N
}
