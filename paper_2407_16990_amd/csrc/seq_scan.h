// rh_state_scan: a selective scan of every stream's state over its tokens.  Both types' sources include this.
//
// Single tokens: the states, 2 * 4 * n bytes a channel, are all that counts.  A lane has four of the up to 128 states of a channel, LN = 1, 2, 4 ... 32
// neighbouring lanes a channel's, so that a wave loads and stores a stretch of memory; what they add to y is summed over them by exchanges inside the wave.
//
// Many tokens: bound by the vector instructions of h = exp2(delta a) h + delta x b, y += c h, of which the power takes twice as long as the four others: 24
// cycles for a wave's 64 states.  A workgroup has CH channels of a stream and goes through its rows, ROWS of them staged in LDS at a time: delta and delta * x of every
// channel, worked out once, b and c in fp32; the next rows' loads are in flight meanwhile.  y takes delta's place.  30 streams of 920 rows, 2048
// channels of 16 states in bf16: 275 us, where the instructions of the recursion alone take 138 and the bytes 89.  A row of a workgroup's 64 channels takes each SIMD 140 cycles by
// count, 94 of them in the recursion, the others mostly in softplus and SiLU.  A CU holds three workgroups (152 registers, 42 KB of LDS), so that the 960 of this call are a round of
// 768 and a quarter of one, at 188 cycles a row and workgroup; one whole round and two (24 and 48 such streams, 193 and 373 us) are at 163 and 160.
// (128 channels a workgroup 295 us where 64 took 286; 32 rows a stage 281, 16 329; registers for four waves a SIMD, some of them spilled, 290.)
// Where streams are few, long ones are cut into chunks that are scanned side by side, twice: from zeros, for what they add to the state behind them, and
// again from the state that those ahead leave.  16384 rows of one stream, 1024 channels: 73 us and 89.  The first launch keeps room in LDS for c, which it does not read: three
// workgroups a CU there too, where its registers would let five in.
// A count of states between the powers of two costs what the next one does, and is masked besides: 30 streams of 250, 1024 channels, 16 states 46 us, 17 to 24 83, 32 73, 48 155, 64 123,
// 65 to 96 340, 128 244.
#pragma once
// us, channels of 16 states in bf16 unless said otherwise.  SCAN_TARGET 2, 3, 4: 16384 rows of one stream, 1024 channels, 155, 160, 163; 37 of up to 2000, 522 of 13 in fp32, 240, 205, 217;
// 8 of 600, 1024, 59.5, 52, 52; 8 of 1000, 1024 of 128, 240, 240, 348; 12 of up to 3000, 1024, 178, 157, 177.  SCAN_LEAST 128: one of 300, 1024, 33.1 for 21.7; one of 1000, 2048, 36.1 for 31.7.
// Cut and whole: one of 230, 1024, 21.8 and 26.8; 8 of 230 30.6 and 31.6; 16 of 230 45 and 34; 30 of 250 65 and 46.
#define SCAN_TARGET 3            // workgroups a CU, or so, that streams are cut for
#define SCAN_LEAST 64            // rows a chunk, at least
#define SCAN_ROWS 64             // rows a stage, at most
#define SCAN_CUT 288             // rows of a stream that is cut, at least
#define SCAN_WHOLE 0x7FFFFFC0    // rows a chunk that no stream has
#include <float.h>
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
    uint32_t* count;             // a counter for every row of ws and workgroup's block of channels, zero between calls
    int32_t channels, n, softplus, chunk, ws_rows;
};

// exp(v), off by an ulp or two: the rounding of v * log2(e) is made up for behind the power of two
__device__ __forceinline__ float scan_exp(float v)
{
    const float hi = v * 1.44269504089f, lo = fmaf(v, 1.92596299e-8f, fmaf(v, 1.44269504089f, -hi));
    const float e = __builtin_amdgcn_exp2f(hi);
    return fmaf(e, lo * 0.69314718056f, e);
}
// log(1 + exp(v)): with w = 1 + e rounded, log(w) * e / (w - 1) makes up for the rounding (Goldberg 1991, theorem 4); where w is 1 the 2^-100 leave e.
// Never below v, which it is where e is infinite and the quotient no number.  A v below -104, whose power is 0 in 32 bits, counts as -104, so that a step masked by -inf or by a
// type's lowest value is 0; by a comparison, which a v that is no number passes.
__device__ __forceinline__ float scan_softplus(float v)
{
    v = v < -104.f ? -104.f : v;
    const float e = scan_exp(v), w = 1.f + e;
    const float l = fmaf(__builtin_amdgcn_logf(w), 0.69314718056f, 0x1p-100f), d = fmaxf(w - 1.f, 0x1p-100f);
    return fmaxf(l * (e * __builtin_amdgcn_rcpf(d)), v);
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
// Four rows' values summed over the LN lanes that lie 64 / LN apart, by exchanges that leave half as many values each time: v[i] then has row scan_row(i).
template <int LN> __device__ __forceinline__ void scan_join(float (&v)[4])
{
    auto halves = [](float& x, float& y, auto rows) {        // of x the lower halves (even rows) of both, of y the upper (odd): their sum
        typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t two;
        two r;
        if constexpr (decltype(rows)::value == 32) r = __builtin_bit_cast(two, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false));
        else r = __builtin_bit_cast(two, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false));
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    };
    auto around = [](float x, auto ctrl) { return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    if constexpr (LN >= 2) { v[0] = halves(v[0], v[1], seq_const<32>()); v[1] = halves(v[2], v[3], seq_const<32>()); }
    if constexpr (LN >= 4) v[0] = halves(v[0], v[1], seq_const<16>());
    if constexpr (LN >= 8) v[0] = around(v[0], seq_const<0x128>());          // 8 lanes around the 16
    if constexpr (LN >= 16) v[0] = around(v[0], seq_const<0x124>());
}
template <int LN> __device__ __forceinline__ int scan_row(int i, int lane) { return LN == 1 ? i : LN == 2 ? 2 * i + (lane >> 5) : (lane >> 4 & 1) * 2 + (lane >> 5); }

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

// a * log2(e), finite where a is: times a delta of 0, a row behind the last among them, it leaves the state as it is
__device__ __forceinline__ f32x4 scan_fade(f32x4 a)
{
    f32x4 v = a * 1.44269504089f;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fabsf(v[e]) == INFINITY ? copysignf(FLT_MAX, v[e]) : v[e];
    return v;
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
    const f32x4 fade = scan_fade(scan_quad<float, FULL>(a.a + at, 4 * j, a.n));
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
// A stream of `len` rows is cut into chunks of equal length, a.chunk rows (whole stages) at most; below one and a half of them, or SCAN_CUT rows, it stays whole.
template <int ROWS> struct scan_cut {
    int32_t size, n;
    __device__ __forceinline__ scan_cut(int32_t len, int32_t chunk)
    {
        if (len < SCAN_CUT || (uint32_t)len < (uint32_t)chunk + (uint32_t)chunk / 2) { size = len; n = len > 0; return; }
        n = (int32_t)(((uint32_t)len + (uint32_t)chunk - 1) / (uint32_t)chunk);
        size = (int32_t)(((uint32_t)len + n - 1) / (uint32_t)n + ROWS - 1) / ROWS * ROWS;
        n = (int32_t)(((uint32_t)len + size - 1) / (uint32_t)size);                         // rounded up to whole stages, fewer may do
    }
};
// The stream that the workgroup's index q falls in, its place in it, and the row of ws where the stream's chunks begin; false where there is none.
// The first launch has every chunk but the last of the streams that are cut; the second has all streams' chunks.
template <int ROWS, bool OUT>
__device__ __forceinline__ bool scan_find(const scan_args& a, int32_t q, int32_t* s_mem, int& b, int32_t& place, int32_t& row)
{
    auto own = [&](int32_t len) { const scan_cut<ROWS> k(len, a.chunk); return OUT ? k.n : k.n < 2 ? 0 : k.n - 1; };
    auto rows = [&](int32_t len) { const scan_cut<ROWS> k(len, a.chunk); return k.n < 2 ? 0 : k.n; };
    if (a.r.n_streams <= 64) {                               // a stream a lane
        streams_lane s, wide;
        int32_t all, unused;
        if (!streams_few(a.r, own, s, all) || q >= all) return false;
        streams_few(a.r, rows, wide, unused);
        b = __builtin_ctzll(__ballot(q >= s.before && q < s.before + s.count));
        place = q - __builtin_amdgcn_readlane(s.before, b);
        row = __builtin_amdgcn_readlane(wide.before, b);
    } else {
        int32_t *s_rows = s_mem + a.r.n_streams + 1, *s_wave = s_rows + a.r.n_streams + 1;
        if (!streams_sums(a.r, s_mem, s_wave, own) || q >= s_mem[a.r.n_streams]) return false;
        streams_sums(a.r, s_rows, s_wave, rows);
        b = __builtin_amdgcn_readfirstlane(streams_find(s_mem, a.r.n_streams, q));
        place = q - __builtin_amdgcn_readfirstlane(s_mem[b]);
        row = __builtin_amdgcn_readfirstlane(s_rows[b]);
    }
    return true;
}

#define SCAN_AHEAD 8             // chunks whose states and sums are in flight
// LN lanes have a channel's states, NS each; E: elements of 16 bytes.
template <typename T, int LN, int NS> struct scan_shape {
    static constexpr int E = 16 / sizeof(T), N = LN * NS, WCH = 64 / LN, CH = 4 * WCH;           // WCH: channels of a wave
    static constexpr int BY_X = 4096 / CH, BY_B = 4096 / N, MOST = SCAN_ROWS;
    static constexpr int ROWS = (BY_X < BY_B ? BY_X : BY_B) < MOST ? (BY_X < BY_B ? BY_X : BY_B) : MOST;     // 32 KB of LDS for delta and delta * x, or for b and c, at most
    static constexpr int PIECES = ROWS * CH / E, NX = (PIECES + 255) / 256;              // of 16 bytes of x, a stage's and a thread's
    static constexpr int QUADS = ROWS * N / 4, NB = (QUADS + 255) / 256;                 // of b, and of c
    static constexpr int DU = CH * 2 + 4, LDS = ROWS * (DU + N * 2) * 4;                 // words of a row of delta and delta * x: four more than it has, so that neighbouring rows begin in other banks
};

// One workgroup's rows of one stream, [first, stop), and CH channels, block blk of them.  OUT: y, and the state behind the stream's last row.  Otherwise what a chunk
// makes of a state of zeros and the sum of its delta; the stream's last such chunk to finish then works out the states that its chunks begin with.
// Lane l of a wave has the states NS * (l / WCH) + ... of the channels l % WCH + ...  The product delta x b goes on the matrix cores, whose 4x4x1 product
// adds to the four states of each of a block's four lanes (channels) the four elements of b times the lane's delta * x: 1 instruction for 4 fused ones and 4 products.
template <typename T, int LN, int NS, bool FULL, bool OUT>
__device__ __forceinline__ void scan_chunk(const scan_args& a, f32x4* s_stage, int b, int32_t place, int32_t ws_row, int32_t chunks, int32_t blk, int32_t first, int32_t stop)
{
    typedef scan_shape<T, LN, NS> S;
    constexpr int E = S::E, CH = S::CH, WCH = S::WCH, N = S::N, ROWS = S::ROWS, NX = S::NX, NB = S::NB, DU = S::DU, Q = NS / 4;
    float* s_du = (float*)s_stage;                           // [row][channel]: delta and delta * x, then y
    float *s_b = s_du + ROWS * DU, *s_c = s_b + ROWS * N;
    int32_t* s_odd = (int32_t*)(s_c + ROWS * N);             // unless FULL: whether any delta * x of the rows in LDS is not finite; of the next ones

    const int t = threadIdx.x, lane = t & 63, cl = (t >> 6) * WCH + lane % WCH, n0 = lane / WCH * NS;
    const int g = (int)seq_quot((uint32_t)blk, a.group_blocks);
    const int c_end = (g + 1) * (int)a.per.d, c_blk = g * (int)a.per.d + (blk - g * (int)a.group_blocks.d) * CH;         // the group's last channel + 1, this block's first
    const int64_t pool = (int64_t)a.channels * a.n;
    float* sums = a.ws + (int64_t)a.ws_rows * a.channels * N;

    // ---- this lane's states, of channel cs (of the last one, and of no account, where the group has no more)
    const int cs = c_blk + cl < c_end ? c_blk + cl : c_end - 1;
    const bool mine = c_blk + cl < c_end;
    const int64_t at = (int64_t)cs * a.n;
    f32x4 h[Q], fade[Q];
    float total = 0.f;
    {
        const int32_t from = chunks < 2 ? streams_slot(a.r, b) : -1;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int n = n0 + 4 * q;
            fade[q] = scan_fade(scan_quad<float, FULL>(a.a + at, n, a.n));
            h[q] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (OUT && chunks > 1) h[q] = *(const f32x4*)(a.ws + ((int64_t)(ws_row + place) * a.channels + cs) * N + n);
            else if (OUT && from >= 0) h[q] = scan_quad<float, FULL>(a.state + from * pool + at, n, a.n);
        }
    }

    // ---- this thread's pieces of the rows: E channels from cc on, the same of every row that it has.  The block's last piece ends where the block does, and so begins
    // inside the one ahead: both give what they share the same values.  A block of fewer channels than a piece goes an element at a time.
    constexpr int PR = CH / E, RX = 256 / PR, RB = 256 / (N / 4);            // pieces a row; rows from a thread's piece, or quad of b, to its next
    // 16 neighbouring threads have pieces of several rows, whose 16 bytes at a time then lie in different banks of LDS: PN pieces of 2 * E words each, of RN rows that begin 4 words apart
    constexpr int PN = PR < 32 / E ? PR : 32 / E, RN = 16 / PN < RX ? 16 / PN : RX;
    const int pc = (t % PN + t / (PN * RN) % (PR / PN) * PN) * E, pr = t / PN % RN + t / (PR * RN) * RN;
    const int cg = c_blk + pc, br = t / (N / 4), bn = t % (N / 4) * 4;
    const bool whole = c_blk + CH <= c_end;
    const bool few = c_end - c_blk < E;
    const int cc = few || cg <= c_end - E ? cg : c_end - E, lc = cc - c_blk, left = c_end - cc;
    float bias[E], skip[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        bias[e] = a.dt_bias && e < left ? a.dt_bias[cc + e] : 0.f;
        skip[e] = OUT && a.skip && e < left ? a.skip[cc + e] : 0.f;
    }
    // where its first piece of a stage's rows lies, and its first quad
    const T *px = (const T*)a.x + ((int64_t)first + pr) * a.x_stride + cc, *pd = (const T*)a.dt + ((int64_t)first + pr) * a.dt_stride + cc;
    const T *pz = (const T*)a.gate + ((int64_t)first + pr) * a.gate_stride + cc;
    const T *pb = (const T*)a.b + ((int64_t)first + br) * a.b_stride + (int64_t)g * a.n, *pq = (const T*)a.c + ((int64_t)first + br) * a.c_stride + (int64_t)g * a.n;
    T* py = (T*)a.y + ((int64_t)first + pr) * a.y_stride + cc;
    struct raw { u32x4 x[NX], dt[NX]; f32x4 b[NB], c[NB]; };
    u32x4 gate[NX];
    auto piece = [&](const T* p) __attribute__((always_inline)) { return few ? row_load<T, E>(p, 0, left < 0 ? 0 : left < E ? left : E - 1) : seq_load<u32x4>(p); };
    auto value = [&](u32x4 w, float (&v)[E]) __attribute__((always_inline)) { row_place<T, E>(w, 0, E, v); };
    // the thread's pieces (quads) of a stage: those of rows that are there; where some are not, behind the last, of the last
    auto each = [&](auto n, auto step, int r0, bool full, int rows, auto f) __attribute__((always_inline)) {
        if (full) {
#pragma unroll
            for (int i = 0; i < decltype(n)::value; ++i) f(i, i * decltype(step)::value);
        } else {
#pragma unroll
            for (int i = 0; i < decltype(n)::value; ++i) f(i, (i * decltype(step)::value + r0 < rows ? i * decltype(step)::value + r0 : rows - 1) - r0);
        }
    };
    const seq_const<NX> nx; const seq_const<NB> nb; const seq_const<RX> rx; const seq_const<RB> rb;
    constexpr bool IDLE = S::PIECES < 256, IDLE_B = S::QUADS < 256;          // threads without a piece, without a quad
    raw in;
    auto load = [&](int rows) __attribute__((always_inline)) {
        if (!IDLE || pr < ROWS) each(nx, rx, pr, rows >= ROWS, rows, [&](int i, int r) { in.x[i] = piece(px + r * a.x_stride); in.dt[i] = piece(pd + r * a.dt_stride); });
        if (!IDLE_B || br < ROWS) each(nb, rb, br, rows >= ROWS, rows, [&](int i, int r) {
            in.b[i] = scan_quad<T, FULL>(pb + r * a.b_stride, bn, a.n);
            if (OUT) in.c[i] = scan_quad<T, FULL>(pq + r * a.c_stride, bn, a.n);
        });
        px += ROWS * a.x_stride; pd += ROWS * a.dt_stride; pb += ROWS * a.b_stride; pq += ROWS * a.c_stride;
    };
    load(stop - first);
    if (a.r.n_streams > 64) __syncthreads();                 // the counts in LDS have been read
    if (!FULL) {
        if (t < 2) s_odd[t] = 0;
        __syncthreads();
    }
    int turn = 0;
    for (int32_t row = first; row < stop; row += ROWS, turn ^= 1) {
        const int rows = stop - row;                         // and those behind the stage's
        const bool full = rows >= ROWS;
        // ---- into LDS; rows behind the last leave the state as it is: delta, delta * x and b are zero
        u32x4 kept[NX];                                      // x, for the skip
        if (!IDLE || pr < ROWS) {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                float x[E], dt[E];
                if (OUT) kept[i] = in.x[i];
                value(in.x[i], x);
                value(in.dt[i], dt);
#pragma unroll
                for (int e = 0; e < E; ++e) dt[e] += bias[e];
                if (a.softplus) {
#pragma unroll
                    for (int e = 0; e < E; ++e) dt[e] = scan_softplus(dt[e]);
                }
                float* to = s_du + (i * RX + pr) * DU + lc * 2;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x[e] *= dt[e];
                    if (!FULL) odd |= !(fabsf(x[e]) < INFINITY);
                }
                if (whole) {                                 // at 16 bytes
#pragma unroll
                    for (int e = 0; e < E; e += 2) *(f32x4*)(to + 2 * e) = f32x4{dt[e], x[e], dt[e + 1], x[e + 1]};
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) *(float2*)(to + 2 * e) = make_float2(dt[e], x[e]);
                }
            }
            if (!FULL && odd) s_odd[turn] = 1;
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            if (IDLE_B && br >= ROWS) break;
            *(f32x4*)(s_b + (i * RB + br) * N + bn) = in.b[i];
            if (OUT) *(f32x4*)(s_c + (i * RB + br) * N + bn) = in.c[i];
        }
        if (!full) {
#pragma unroll
            for (int i = 0; i < NX; ++i)
                if (i * RX + pr >= rows && (!IDLE || pr < ROWS))
#pragma unroll
                    for (int e = 0; e < E; ++e) *(float2*)(s_du + (i * RX + pr) * DU + (lc + e) * 2) = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NB; ++i)
                if (i * RB + br >= rows && (!IDLE_B || br < ROWS)) *(f32x4*)(s_b + (i * RB + br) * N + bn) = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        __syncthreads();
        // ---- the next rows' loads, and these rows' gate
        if (OUT && a.gate) {
            if (!IDLE || pr < ROWS) each(nx, rx, pr, full, rows, [&](int i, int r) { gate[i] = piece(pz + r * a.gate_stride); });
            pz += ROWS * a.gate_stride;
        }
        if (rows > ROWS) load(rows - ROWS);
        // ---- the rows
        auto four = [&](int r0, auto masked) __attribute__((always_inline)) {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i;
                const float2 du = *(const float2*)(s_du + r * DU + cl * 2);
                float sum = 0.f;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const float bq = s_b[r * N + n0 + 4 * q + lane % 4];
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = h[q][e] * __builtin_amdgcn_exp2f(du.x * fade[q][e]);
                    v = __builtin_amdgcn_mfma_f32_4x4x1f32(bq, du.y, v, 0, 0, 0);
                    if constexpr (decltype(masked)::value) {                // states that are none: an infinite delta * x times their zero
#pragma unroll
                        for (int e = 0; e < 4; ++e) if (n0 + 4 * q + e >= a.n) v[e] = 0.f;
                    }
                    if constexpr (OUT) {
                        const f32x4 cq = *(const f32x4*)(s_c + r * N + n0 + 4 * q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum = q + e ? fmaf(cq[e], v[e], sum) : cq[e] * v[e];
                    }
                    h[q] = v;
                }
                y[i] = sum;
                if (!OUT) total += du.x;
            }
            if constexpr (OUT) {
                scan_join<LN>(y);
#pragma unroll
                for (int i = 0; i < (LN < 4 ? 4 / LN : 1); ++i) s_du[(r0 + scan_row<LN>(i, lane)) * DU + cl * 2] = y[i];
            }
        };
        const int some = full ? ROWS : rows;
        __builtin_amdgcn_s_setprio(1);                       // ahead of waves that stage: 37 ragged streams 216 -> 205 us, 64 of 64 states 102 -> 98
        if (!FULL && s_odd[turn]) for (int r0 = 0; r0 < some; r0 += 4) four(r0, seq_const<1>());
        else for (int r0 = 0; r0 < some; r0 += 4) four(r0, seq_const<0>());
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();
        if (!FULL && t == 0) s_odd[turn] = 0;                // the rows after the next write it again, behind a barrier
        // ---- y: the thread's own pieces, which it alone fills with the next rows (but for the block's last, see below)
        if constexpr (OUT) {
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                if (i * RX + pr >= some) continue;
                float y[E], z[E];
                const float* from = s_du + (i * RX + pr) * DU + lc * 2;
                if (whole) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) { const f32x4 v = *(const f32x4*)(from + 2 * e); y[e] = v[0]; y[e + 1] = v[2]; }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] = from[2 * e];
                }
                if (a.skip) {
                    value(kept[i], z);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] = fmaf(skip[e], z[e], y[e]);
                }
                if (a.gate) {
                    value(gate[i], z);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] *= seq_silu(z[e]);
                }
                if (cg < c_end) row_store<T, E>(py + i * RX * a.y_stride, few ? left : E, y);
            }
            py += ROWS * a.y_stride;
            if (!whole) __syncthreads();         // pieces that share places: none is filled before all have been read
        }
    }
    if constexpr (OUT) {                                     // ---- the state behind the last row
        const int32_t to = place == chunks - 1 ? streams_into(a.r, b) : -1;
        if (to < 0 || !mine) return;
#pragma unroll
        for (int q = 0; q < Q; ++q) scan_put<FULL>(a.state + to * pool + at, n0 + 4 * q, a.n, h[q]);
    } else {
        // ---- what the chunk leaves.  The chunks of a stream sit on eight XCDs with an L2 each: stored through with relaxed atomics of the device's scope, loaded past
        // the L2 by the one that finishes last, and acknowledged before the chunk is counted.
        struct two { uint64_t u[2]; };
        auto state_at = [&](int32_t chunk, int q) {          // a row's place is the same for all lanes, theirs in it 32 bits
            return (float*)((char*)(a.ws + (int64_t)(ws_row + chunk) * a.channels * N) + (uint32_t)((cs * N + n0 + 4 * q) * 4));
        };
        auto sum_at = [&](int32_t chunk) { return (uint32_t*)((char*)(sums + (int64_t)(ws_row + chunk) * a.channels) + (uint32_t)(cs * 4)); };
        if (mine) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const two w = __builtin_bit_cast(two, h[q]);
                uint64_t* p = (uint64_t*)state_at(place, q);
                __hip_atomic_store(p, w.u[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(p + 1, w.u[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            if (n0 == 0) __hip_atomic_store(sum_at(place), __float_as_uint(total), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        int32_t* s_last = (int32_t*)s_stage;                 // what LDS held has been read
        __syncthreads();
        if (t == 0) {
            uint32_t* count = a.count + (int64_t)ws_row * a.blocks.d + blk;
            const bool last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)chunks - 2;
            if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *s_last = last;
        }
        __syncthreads();
        if (!*s_last || !mine) return;
        // ---- h = exp(a * sum of delta) h + what the chunk makes of zeros, chunk after chunk, in the place of the latter: the states that chunks begin with
        const int32_t from = streams_slot(a.r, b);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (from >= 0) v = scan_quad<float, FULL>(a.state + from * pool + at, n0 + 4 * q, a.n);
            for (int32_t c0 = 0; c0 < chunks; c0 += SCAN_AHEAD) {
                two add[SCAN_AHEAD];
                uint32_t sum[SCAN_AHEAD];
#pragma unroll
                for (int i = 0; i < SCAN_AHEAD; ++i) {
                    const int32_t k = c0 + i < chunks - 1 ? c0 + i : 0;                  // the last chunk leaves nothing
                    const uint64_t* p = (const uint64_t*)state_at(k, q);
                    add[i].u[0] = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    add[i].u[1] = __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    sum[i] = __hip_atomic_load(sum_at(k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
#pragma unroll
                for (int i = 0; i < SCAN_AHEAD; ++i) {
                    if (c0 + i >= chunks) break;
                    *(f32x4*)state_at(c0 + i, q) = v;
                    const f32x4 more = __builtin_bit_cast(f32x4, add[i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // As if no row's power were 0 or infinite, whatever all of them make: in two halves, which neither are, an infinite state stays infinite,
                        // one of zeros zero, and a small one may grow by more than 2^128.  Where a row's own is, the rows one after the other make an infinite state, or one of
                        // zeros, no number instead.
                        float f = __builtin_amdgcn_exp2f(0.5f * __uint_as_float(sum[i]) * fade[q][e]);
                        f = f == 0.f ? 0x1p-149f : f > FLT_MAX ? FLT_MAX : f;
                        v[e] = fmaf(f, f * v[e], more[e]);
                        if (!FULL && n0 + 4 * q + e >= a.n) v[e] = 0.f;                  // a state that is none: an infinite sum times its zero
                    }
                }
            }
        }
    }
}

template <typename T, int LN, int NS, bool FULL, bool OUT>
__global__ __launch_bounds__(256, 2) void k_seq_scan(scan_args a)
{
    constexpr int ROWS = scan_shape<T, LN, NS>::ROWS;
    extern __shared__ f32x4 s_stage[];
    const uint32_t item = seq_quot(blockIdx.x, a.blocks), blk = blockIdx.x - item * a.blocks.d;
    int b;
    int32_t place, ws_row, begin, end;
    if (!scan_find<ROWS, OUT>(a, (int32_t)item, (int32_t*)s_stage, b, place, ws_row)) return;
    streams_rows(a.r, b, begin, end);
    const scan_cut<ROWS> cut(end - begin, a.chunk);
    const int32_t first = begin + place * cut.size, stop = end - first < cut.size ? end : first + cut.size;
    scan_chunk<T, LN, NS, FULL, OUT>(a, s_stage, b, place, ws_row, cut.n, (int32_t)blk, first, stop);
}

// a launch has fewer than 2^32 threads
static rh_status scan_fits(rh_ctx* ctx, const scan_args& a, int64_t workgroups)
{
    if (workgroups > 0xFFFFFF) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_scan: %d rows of %d streams and %d channels are %lld workgroups (at most %d)", a.r.n_rows, a.r.n_streams, a.channels, (long long)workgroups, 0xFFFFFF);
    return RH_OK;
}

template <typename T, int LN, bool FULL>
static hipError_t launch_scan(rh_ctx* ctx, scan_args& a, rh_status* failed)
{
    constexpr int WL = LN > 16 ? 16 : LN, NS = 4 * LN / WL;
    typedef scan_shape<T, WL, NS> S;
    const int groups = a.channels / (int)a.per.d;
    const int64_t wide = (a.channels + 256 / LN - 1) / (256 / LN);           // workgroups of one channel a thread
    if (!a.r.offsets) {
        a.blocks = seq_make_div((uint32_t)wide);
        // four streams a thread and one, us: 512 of 4096 channels 57 and 71, 256 of 1024 10.0 and 9.9, 64 of 2048 7.1 and 6.2, 8 of 1024 4.9 and 3.9
        const bool four = wide * a.r.n_rows >= 16 * (int64_t)ctx->n_cu;
        const int64_t workgroups = (four ? ((int64_t)a.r.n_rows + 3) / 4 : a.r.n_rows) * wide;
        if ((*failed = scan_fits(ctx, a, workgroups)) != RH_OK) return hipSuccess;
        if (four) hipLaunchKernelGGL((k_seq_scan_step<T, LN, FULL, 4>), dim3((unsigned)workgroups), dim3(256), 0, ctx->stream, a);
        else hipLaunchKernelGGL((k_seq_scan_step<T, LN, FULL, 1>), dim3((unsigned)workgroups), dim3(256), 0, ctx->stream, a);
        return hipGetLastError();
    }
    const int group_blocks = ((int)a.per.d + S::CH - 1) / S::CH;
    const int64_t blocks = (int64_t)groups * group_blocks;
    a.blocks = seq_make_div((uint32_t)blocks);
    a.group_blocks = seq_make_div((uint32_t)group_blocks);
    // Rows a chunk: enough workgroups for the GPU where streams are few, and no more states than the scratch memory holds.  Nothing is cut where the channels alone are enough:
    // so (3/2 rows / chunk + 1) * blocks, the counters that there may be, stay below 4.5 + 4 a CU of the 16.
    const int64_t room = SCAN_ROOM(ctx) / ((int64_t)a.channels * (S::N + 1));
    const int64_t least = room > 0 ? (int64_t)a.r.n_rows * 3 / (2 * room) + 1 : SCAN_WHOLE;
    int64_t chunk = (int64_t)a.r.n_rows * blocks / (SCAN_TARGET * ctx->n_cu);
    chunk = chunk < SCAN_LEAST ? SCAN_LEAST : chunk;
    chunk = chunk < least ? least : chunk;
    chunk = (chunk + S::ROWS - 1) / S::ROWS * S::ROWS;
    a.chunk = (int32_t)(chunk > SCAN_WHOLE || blocks > 4 * ctx->n_cu ? SCAN_WHOLE : chunk);
    const bool cut = a.r.n_rows >= SCAN_CUT && 2 * (int64_t)a.r.n_rows >= 3 * (int64_t)a.chunk;        // otherwise no stream can be as long
    a.ws_rows = cut ? (int32_t)((int64_t)a.r.n_rows * 3 / (2 * (int64_t)a.chunk)) + 1 : 0;
    const size_t counts = a.r.n_streams > 64 ? (2 * (a.r.n_streams + 1) + STREAMS_T / 64) * sizeof(int32_t) : 0, stage = S::LDS + (FULL ? 0 : 2 * sizeof(int32_t));
    const size_t lds = stage > counts ? stage : counts;
    const int64_t workgroups = ((int64_t)a.r.n_rows / a.chunk + a.r.n_streams) * blocks;      // as many as any offsets give; the first launch has no more
    if ((*failed = scan_fits(ctx, a, workgroups)) != RH_OK) return hipSuccess;
    if (cut) {
        rh_status st = seq_counters(ctx);
        if (st == RH_OK) st = seq_scratch(ctx);
        if (st != RH_OK) { *failed = st; return hipSuccess; }
        a.ws = (float*)ctx->seq_ws; a.count = ctx->seq_cnt;
    }
    if (cut) {
        hipLaunchKernelGGL((k_seq_scan<T, WL, NS, FULL, false>), dim3((unsigned)(((int64_t)a.r.n_rows / a.chunk + 1) * blocks)), dim3(256), lds, ctx->stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_seq_scan<T, WL, NS, FULL, true>), dim3((unsigned)workgroups), dim3(256), lds, ctx->stream, a);
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
