// rh_matvec_packed: products of a few rows with weights in 4 bits that share a scale by 32.
//
// Bound by the weights' bytes: a wave streams them from memory into the matrix operand, 16 outputs a product, and the rows x are the
// other operand, out of LDS, where a workgroup lays them once for all the outputs that it goes through.  A lane's 16 bytes are the 32 codes of
// one block, so that one scale byte goes with them.
//   bf16 rows   8 codes at a time become bf16 values, their block's scale included (a conversion of the hardware; exact)
//   fp32 rows   the same against x cut into three bf16 parts, which together are x exactly: products of full precision at three
//               products of the 16-bit rate, where the fp32 rate is a sixteenth of it
//   e4m3 rows   as bf16 rows, which hold them exactly.  (The scaled product of 8-bit and 4-bit values would take codes, scales and rows as they
//               are - 10.1 us for 16 x 16384 x 4096 - but keeps fewer than 32 bits of its partial sums: two pairs of +-448 that cancel in a row of 8192 small terms
//               left 1.2 where the sum is -0.03.)
// A workgroup's waves share out its tiles of outputs and the inner index (KS waves a tile, summed in LDS in order), so that few outputs
// still use every wave; where x is long or the tiles are few, workgroups share the inner index too, and the last of them adds up their sums, in their order.
// 16 x 16384 x 4096, e4m3 rows: 11.6 us, 3.1 TB/s of weights; 7.0 at a copy's rate, about 2 until the first bytes are there, the rest x.  1 x 1024 x 510,
// fp32: 4.1, hardly more than an empty launch (2.5) and one way to memory.
#include "seq_common.h"

struct matvec_args {
    const void* x;
    const uint8_t *w, *w_scale;
    int64_t x_stride;
    int32_t rows, outs, ins, blocks;
    int32_t tiles, ks, tw;       // tiles of outputs; waves a tile; tiles a workgroup at a time
    int32_t threads;             // of a workgroup
    int32_t quads, slice, chunk; // stretches of 512 of the inner index: all, a workgroup's, and as many as x lies in LDS for at a time
    const float* x_scale;
    void* y;
    int64_t y_stride;
    int32_t relu, y_f32;
    uint64_t* part;              // sums of slices of the inner index [group of rows][tile][R * MT][slice][half][lane]
    uint32_t* count;             // [group of rows][workgroup of a slice]
    int32_t slices;
};

#define MATVEC_WAVES(XT, MT) (MT == 1 && XT != RH_T_F32 ? 16 : 8)       // of a workgroup, one a CU; the others' registers allow eight
#define MATVEC_PIECE 8           // elements of x in 16 bytes of LDS
#define MATVEC_LDS (160 * 1024)
#define MATVEC_HUGE 252          // scales from here on can take a code past the largest bf16 number

template <int XT> struct matvec_kind;
template <> struct matvec_kind<RH_T_F32> { typedef float T; static constexpr int PARTS = 3; };
template <> struct matvec_kind<RH_T_BF16> { typedef __bf16 T; static constexpr int PARTS = 1; };
template <> struct matvec_kind<RH_T_E4M3> { typedef uint8_t T; static constexpr int PARTS = 1; };

// x = the sum of three bf16 numbers, for any finite x: cut off, not rounded, so that none passes the largest
__device__ __forceinline__ void matvec_cut(float x, uint32_t (&part)[3])
{
    const uint32_t u = __float_as_uint(x);
    const bool finite = (u & 0x7F800000u) != 0x7F800000u;
    part[0] = x != x ? 0x7FC0u : u >> 16;
    const float r = finite ? x - __uint_as_float(u & 0xFFFF0000u) : 0.f;
    part[1] = __float_as_uint(r) >> 16;
    part[2] = __float_as_uint(r - __uint_as_float(__float_as_uint(r) & 0xFFFF0000u)) >> 16;
}

// 8 codes (the bytes of c, low half first) times 2^(scale - 127) as bf16
__device__ __forceinline__ bf16x8 matvec_wide(uint32_t c, uint32_t scale)
{
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const float f = __uint_as_float(scale << 23);
    union { bf16x2 two[4]; bf16x8 all; } r;
    r.two[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 0);
    r.two[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 1);
    r.two[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 2);
    r.two[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 3);
    return r.all;
}
// The value of a code without its block's scale
__device__ __forceinline__ float matvec_code(uint32_t code)
{
    const uint32_t m = code & 7;
    const float f = m < 2 ? 0.5f * (float)m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
    return code & 8 ? -f : f;
}

// SPLIT: the inner index is cut into slices; ENDS: it is no multiple of 512 (what the others need not look at costs them up to 0.8 us of 14)
template <int XT, int MT, int R, bool SPLIT, bool ENDS>
__global__ __launch_bounds__(64 * MATVEC_WAVES(XT, MT)) void k_seq_matvec(matvec_args a)
{
    typedef matvec_kind<XT> K;
    typedef typename K::T T;
    constexpr int PARTS = K::PARTS, PIECE = MATVEC_PIECE, PER_STEP = 128 / PIECE;      // 16-byte pieces of a row in a step of 128
    extern __shared__ uint4 s_mem[];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, c = lane & 15, j = lane >> 4;
    const int tw = wave / a.ks, ks = wave % a.ks;
    const int qb = SPLIT ? blockIdx.z * a.slice : 0, qe = SPLIT && qb + a.slice < a.quads ? qb + a.slice : a.quads;       // the workgroup's slice
    const int m0 = blockIdx.y * 16 * MT, M = a.rows - m0 < 16 * MT ? a.rows - m0 : 16 * MT, P = M | 1;
    // x in LDS: pieces of 16 bytes, [part][step][as the lanes of a product read them][row]; an odd number P of rows, or neighbouring
    // pieces of a row would be written to the same banks (16 x 4096 x 4096, bf16 rows: 8.4 -> 6.9 us)
    const int part_pieces = a.chunk * 4 * PER_STEP * P;
    u32x4* xs = (u32x4*)s_mem;
    // the waves' sums [wave][R * MT][lane]: behind x, or in its place where x does not lie here as a whole
    f32x4* s_sum = (f32x4*)(a.chunk < a.slice ? xs : xs + PARTS * part_pieces);

    constexpr int W = PIECE * sizeof(T) / 4;                 // words of a piece in memory
    auto put = [&](int m, int p, const uint32_t* v) {        // piece p of row m
        // lane quarter j of the e-th product of a step reads block j's piece e
        const int step = p / PER_STEP, in = p % PER_STEP;
        u32x4* to = xs + (step * PER_STEP + in % 4 * 4 + in / 4) * P + m;
        if constexpr (XT == RH_T_F32) {
            uint32_t w[3][4];
#pragma unroll
            for (int d = 0; d < 8; d += 2) {
                uint32_t lo[3], hi[3];
                matvec_cut(__uint_as_float(v[d]), lo);
                matvec_cut(__uint_as_float(v[d + 1]), hi);
#pragma unroll
                for (int s = 0; s < 3; ++s) w[s][d / 2] = lo[s] | hi[s] << 16;
            }
#pragma unroll
            for (int s = 0; s < 3; ++s) to[s * part_pieces] = u32x4{w[s][0], w[s][1], w[s][2], w[s][3]};
        } else if constexpr (W == 4) *to = u32x4{v[0], v[1], v[2], v[3]};
        else *to = u32x4{seq_e4m3_pair<false>(v[0]), seq_e4m3_pair<true>(v[0]), seq_e4m3_pair<false>(v[1]), seq_e4m3_pair<true>(v[1])};
    };
    auto get = [&](const T* from, uint32_t* v) {             // a whole piece
        if constexpr (W == 2) { const uint2 u = seq_load<uint2>(from); v[0] = u.x; v[1] = u.y; }
        else
#pragma unroll
            for (int d = 0; d < W; d += 4) {
                const u32x4 u = seq_load<u32x4>((const uint32_t*)from + d);
                v[d] = u[0]; v[d + 1] = u[1]; v[d + 2] = u[2]; v[d + 3] = u[3];
            }
    };
    // a row's end that has been loaded as a whole piece, from `by` elements ahead and so still in the row, moved to its place, with zeros behind
    auto settle = [&](uint32_t (&v)[W], int by) {
        const int b = by * (int)sizeof(T);                   // bytes
#pragma unroll
        for (int d = W / 2; d; d /= 2)
#pragma unroll
            for (int k = 0; k < W; ++k) v[k] = b & 4 * d ? k + d < W ? v[k + d] : 0 : v[k];
        if constexpr (sizeof(T) < 4)
#pragma unroll
            for (int k = 0; k < W; ++k) v[k] = __builtin_amdgcn_alignbyte(k + 1 < W ? v[k + 1] : 0, v[k], b & 3);
    };
    // piece p of row m, which may hold the row's end, or lie behind it
    auto get_end = [&](int q0, int m, int p, uint32_t (&v)[W]) {
        const T* from = (const T*)a.x + (m0 + m) * a.x_stride;
        const int e = q0 * 512 + p * PIECE, n = a.ins - e;
        if (n >= PIECE) get(from + e, v);
        else if (n > 0) {
            if (XT != RH_T_F32 && a.ins >= PIECE) { get(from + a.ins - PIECE, v); settle(v, PIECE - n); }
            else
#pragma unroll
                for (int d = 0; d < PIECE; ++d) {            // eight words at most, or a row shorter than a piece
                    const uint32_t bits = d >= n ? 0 : sizeof(T) == 4 ? *(const uint32_t*)(from + e + d) : sizeof(T) == 2 ? *(const uint16_t*)(from + e + d) : *(const uint8_t*)(from + e + d);
                    v[d * sizeof(T) / 4] |= bits << (8 * sizeof(T) * (d % (4 / sizeof(T))));
                }
        }
    };
    auto stage = [&](int q0, int nq) {
        const int per_row = nq * 4 * PER_STEP;               // pieces of a row in LDS
        int whole = per_row;                                 // and those that the first loop takes
        if constexpr (ENDS) {
            const int left = (a.ins - q0 * 512) / PIECE;
            whole = left >= per_row ? per_row : XT == RH_T_F32 ? 0 : left;
        }
        const int all = whole * M;
        // i / whole by a product: (i + 1/2) / whole is at least 1 / (2 whole) away from a whole number, and the product's error, below
        // 2^-21 of it, stays below that, since i < 2^14 (what fits the LDS)
        const float inverse = __builtin_amdgcn_rcpf((float)whole);
        constexpr int AHEAD = 4;                             // pieces of a thread in flight
        for (int first = t; first < all; first += AHEAD * a.threads) {
            uint32_t v[AHEAD][W];
            int m[AHEAD], p[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {                // behind the last: the last again
                int i = first + k * a.threads;
                i = i < all ? i : all - 1;
                m[k] = (int)(((float)i + 0.5f) * inverse); p[k] = i - m[k] * whole;
                get((const T*)a.x + (m0 + m[k]) * a.x_stride + q0 * 512 + p[k] * PIECE, v[k]);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                // fp32 rows, whose pieces take time to cut: only once (1 x 1024 x 512: 5.2 -> 4.7 us; bf16 rows are slower so, 64 x 1024 x 512 5.6 -> 6.3)
                if (XT == RH_T_F32 && first + k * a.threads >= all) break;
                put(m[k], p[k], v[k]);
            }
        }
        if constexpr (ENDS) {
            // Rows that end in here: the piece with a row's end, and zeros behind it, beginning with the last threads; of fp32 rows all pieces, one at a
            // time (1 x 1024 x 510: 4.6 us, as the others 5.2; those so: 16 x 4096 x 4090, bf16, 10.0, as they are 7.7).
            const int rest = per_row - whole;
            const float inv = __builtin_amdgcn_rcpf((float)rest);
            for (int i = XT == RH_T_F32 ? t : a.threads - 1 - t; i < rest * M; i += a.threads) {
                const int m = (int)(((float)i + 0.5f) * inv), p = whole + i - m * rest;
                uint32_t v[W] = {};
                get_end(q0, m, p, v);
                put(m, p, v);
            }
        }
    };

    // ---- a wave's weights: tile by tile of outputs, of each its share of the stretches of every chunk
    struct place { int tile, q0, q, end; };                  // q0: the chunk's first stretch; q, end: of the wave's share, in the chunk
    auto share = [&](place& p) {
        const int n = qe - p.q0 < a.chunk ? qe - p.q0 : a.chunk, each = (n + a.ks - 1) / a.ks;
        p.q = ks * each;
        p.end = p.q + each < n ? p.q + each : n;
    };
    const int tile_step = gridDim.x * a.tw;
    // the next stretch, of this chunk or of a later chunk or tile; false: there is none
    auto advance = [&](place& p) -> bool {
        ++p.q;
        while (p.q >= p.end) {
            p.q0 += a.chunk;
            if (p.q0 >= qe) { p.q0 = qb; p.tile += tile_step; }
            if (p.tile >= a.tiles) return false;
            share(p);
        }
        return true;
    };
    struct weights { u32x4 code[R][4]; u32x4 scale[R]; };
    auto load = [&](const place& p, weights& w) {
        const int quad = p.q0 + p.q;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            int n = (p.tile * R + r) * 16 + c;
            n = n < a.outs ? n : a.outs - 1;
            const int b0 = quad * 16;                        // the stretch's first block
            const uint8_t* code = a.w + ((int64_t)n * a.blocks + b0) * 16;
            const uint8_t* scale = a.w_scale + (int64_t)n * a.blocks + b0;
            if (!ENDS || b0 + 16 <= a.blocks) {
#pragma unroll
                for (int s = 0; s < 4; ++s) w.code[r][s] = *(const u32x4*)(code + (4 * s + j) * 16);
                w.scale[r] = seq_load<u32x4>(scale);
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const bool in = b0 + 4 * s + j < a.blocks;   // a block that is none: codes of zero, a scale of one
                    const u32x4 v = *(const u32x4*)(in ? code + (4 * s + j) * 16 : a.w);
                    w.code[r][s] = in ? v : u32x4{0, 0, 0, 0};
                    // of the scales, the lane's own (one by one with the others of the word: 16 x 1024 x 1000, e4m3 rows, 8.5 us)
                    const uint32_t e = scale[in ? 4 * s + j : 0];
                    w.scale[r][s] = (in ? e : 127) << (8 * j);
                }
            }
        }
    };

    f32x4 acc[R][MT];
    int mrow[MT];                                            // rows that are none read row 0
#pragma unroll
    for (int i = 0; i < MT; ++i) mrow[i] = j * P + (16 * i + c < M ? 16 * i + c : 0);

    auto multiply = [&](const weights& w, int q) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const u32x4* x = xs + (q * 4 + s) * PER_STEP * P;
            uint32_t scale[R];
            bool huge = false;
#pragma unroll
            for (int r = 0; r < R; ++r) { scale[r] = w.scale[r][s] >> (8 * j) & 255; huge |= scale[r] >= MATVEC_HUGE; }
            if (!__any(huge)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    bf16x8 wa[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) wa[r] = matvec_wide(w.code[r][s][e], scale[r]);
#pragma unroll
                    for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            const bf16x8 xb = __builtin_bit_cast(bf16x8, x[p * part_pieces + e * 4 * P + mrow[i]]);
#pragma unroll
                            for (int r = 0; r < R; ++r) acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[r], xb, acc[r][i], 0, 0, 0);
                        }
                }
            } else {
                // A block whose codes bf16 cannot hold: this step a term at a time in 32 bits, where blocks of any other scale keep their values beside it.  Terms of
                // such blocks are summed by 2^-8.  The lane that has output 4*j + e of a product has its block b's codes in lane 16*b + 4*j + e.  (Seldom
                // or never reached: written for few registers.)
#pragma unroll 1
                for (int e = 0; e < 4; ++e) {
                    float plain[R][MT] = {}, huge8[R][MT] = {};
#pragma unroll 1
                    for (int at = 0; at < 16; ++at) {
                        const int b = at >> 2, e8 = at & 3;  // block, and eight of its codes
                        uint32_t code[R], by[R];
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const u32x4 all = w.code[r][s];
                            code[r] = (uint32_t)__shfl((int)(e8 == 0 ? all[0] : e8 == 1 ? all[1] : e8 == 2 ? all[2] : all[3]), 16 * b + 4 * j + e);
                            by[r] = (uint32_t)__shfl((int)scale[r], 16 * b + 4 * j + e);
                        }
#pragma unroll 1
                        for (int n = 0; n < 8; ++n) {
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                float v = 0.f;
#pragma unroll
                                for (int p = PARTS - 1; p >= 0; --p)
                                    v += __uint_as_float((uint32_t)((const uint16_t*)&x[p * part_pieces + (e8 * 4 + b) * P + mrow[i] - j * P])[n] << 16);
#pragma unroll
                                for (int r = 0; r < R; ++r) {
                                    const bool is_huge = by[r] >= MATVEC_HUGE;
                                    const float f = by[r] == 255 ? __builtin_nanf("") : matvec_code(code[r] >> (4 * n));
                                    const float term = __builtin_amdgcn_ldexpf(f * v, (int)by[r] - (is_huge ? 135 : 127));
                                    plain[r][i] += is_huge ? 0.f : term;
                                    huge8[r][i] += is_huge ? term : 0.f;
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[r][i][k] += k == e ? plain[r][i] + huge8[r][i] * 256.f : 0.f;
                }
            }
        }
    };

    auto write = [&](int tile, int r, int i, f32x4 v) {
        const int m = 16 * i + c, n = (tile * R + r) * 16 + 4 * j;
        if (m >= M || n >= a.outs) return;
        if (a.x_scale) v *= a.x_scale[m0 + m];
        if (a.relu) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
        }
        const int64_t at = (m0 + m) * a.y_stride + n;
        if (a.y_f32) {
            float* o = (float*)a.y + at;
            if (n + 4 <= a.outs) seq_store(o, v);
            else for (int e = 0; n + e < a.outs; ++e) o[e] = v[e];
        } else {
            __bf16* o = (__bf16*)a.y + at;
            if (n + 4 <= a.outs) seq_store(o, make_uint2(seq_pack_bf16(v[0], v[1]), seq_pack_bf16(v[2], v[3])));
            else for (int e = 0; n + e < a.outs; ++e) o[e] = (__bf16)v[e];
        }
    };

    struct two { uint64_t u[2]; };
    auto part = [&](int tile, int z, int r, int i) {
        return a.part + (((((size_t)blockIdx.y * a.tiles + tile) * R + r) * MT + i) * a.slices + z) * 128 + lane;
    };

    place at = {(int)blockIdx.x * a.tw + tw, qb, 0, 0};
    weights now, next;
    const bool idle = tw >= a.tw;                            // waves that only help to lay x out
    bool have = !idle && at.tile < a.tiles;
    if (have) {
        share(at);
        if (at.q >= at.end) { at.q = at.end; have = advance(at); }
        if (have) load(at, now);
    }
    int staged = -1;                                         // the chunk that is in LDS
    for (int first = blockIdx.x * a.tw; first < a.tiles; first += tile_step) {     // the same rounds for every wave
        const int tile = first + tw;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q0 = qb; q0 < qe; q0 += a.chunk) {
            if (staged != q0) {
                if (staged >= 0) __syncthreads();
                stage(q0, qe - q0 < a.chunk ? qe - q0 : a.chunk);
                __syncthreads();
                staged = q0;
            }
            while (have && at.tile == tile && at.q0 == q0) {
                const int q = at.q;
                have = advance(at);
                if (have) load(at, next);
                multiply(now, q);
                now = next;
            }
        }
        if (a.ks > 1) {
            __syncthreads();                                 // the sums of the round before have been read
            if (ks && !idle) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < MT; ++i) s_sum[(wave * R * MT + r * MT + i) * 64 + lane] = acc[r][i];
            }
            __syncthreads();
            if (!ks && !idle) {
                for (int k = 1; k < a.ks; ++k)
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int i = 0; i < MT; ++i) acc[r][i] += s_sum[((wave + k) * R * MT + r * MT + i) * 64 + lane];
            }
            if (a.chunk < a.slice) staged = a.quads;         // no chunk: the sums lie there
        }
        if (ks || idle || tile >= a.tiles) continue;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if constexpr (!SPLIT) write(tile, r, i, acc[r][i]);
                else if (16 * i + c < M) {
                    const two v = __builtin_bit_cast(two, acc[r][i]);
                    uint64_t* p = part(tile, blockIdx.z, r, i);
                    __hip_atomic_store(p, v.u[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __hip_atomic_store(p + 64, v.u[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            }
    }
    if constexpr (!SPLIT) return;
    // ---- the slices' sums: the workgroup that comes last with its tiles adds them up, in the slices' order.  Slices run on several XCDs: sums are stored
    // through and loaded past the L2, and acknowledged before they are counted.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* s_last = (uint32_t*)s_mem;
    if (t == 0) {
        uint32_t* count = a.count + blockIdx.y * gridDim.x + blockIdx.x;
        const bool last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.slices - 1;
        if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = last;
    }
    __syncthreads();
    if (!*s_last) return;
    const int rounds = (a.tiles - (int)blockIdx.x * a.tw + tile_step - 1) / tile_step, vectors = rounds * a.tw * R * MT;
    auto join = [&](auto ahead) __attribute__((always_inline)) {
        constexpr int Z = decltype(ahead)::value, N = 16 / Z;                  // a wave loads Z slices of N vectors at a time
        for (int n0 = wave * N; n0 < vectors; n0 += (a.threads >> 6) * N) {
            f32x4 sum[N] = {};
            for (int z = 0; z < a.slices; z += Z) {
                two v[N][Z];
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const int n = n0 + q, nth = n / (R * MT);
                    int tile = blockIdx.x * a.tw + nth / a.tw * tile_step + nth % a.tw;
                    tile = tile < a.tiles ? tile : a.tiles - 1;
#pragma unroll
                    for (int k = 0; k < Z; ++k) {
                        const uint64_t* p = part(tile, z + k < a.slices ? z + k : z, n / MT % R, n % MT);
                        v[q][k].u[0] = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        v[q][k].u[1] = __hip_atomic_load(p + 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                }
#pragma unroll
                for (int q = 0; q < N; ++q)
#pragma unroll
                    for (int k = 0; k < Z; ++k)
                        if (z + k < a.slices) sum[q] += __builtin_bit_cast(f32x4, v[q][k]);
            }
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const int n = n0 + q, nth = n / (R * MT), tile = blockIdx.x * a.tw + nth / a.tw * tile_step + nth % a.tw;
                if (n < vectors && tile < a.tiles) write(tile, n / MT % R, n % MT, sum[q]);
            }
        }
    };
    if (a.slices <= 4) join(seq_const<4>()); else if (a.slices <= 8) join(seq_const<8>()); else join(seq_const<16>());
}

template <int XT, int MT, int R>
static hipError_t launch_matvec(rh_ctx* ctx, matvec_args a)
{
    typedef matvec_kind<XT> K;
    static bool attr_done[RH_MAX_DEVICES] = {};              // the attribute is per device
    if (!attr_done[ctx->device]) {
        for (const void* f : {(const void*)k_seq_matvec<XT, MT, R, false, false>, (const void*)k_seq_matvec<XT, MT, R, true, false>,
                              (const void*)k_seq_matvec<XT, MT, R, false, true>, (const void*)k_seq_matvec<XT, MT, R, true, true>}) {
            const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, MATVEC_LDS);
            if (e != hipSuccess) return e;
        }
        attr_done[ctx->device] = true;
    }
    const int M = a.rows < 16 * MT ? a.rows : 16 * MT, quad = K::PARTS * 512 / MATVEC_PIECE * 16 * (M | 1);       // bytes of x in LDS, of a stretch
    constexpr int WAVES = MATVEC_WAVES(XT, MT), SUMS = WAVES * R * MT * 64 * (int)sizeof(f32x4);
    const int gy = (a.rows + 16 * MT - 1) / (16 * MT);
    a.quads = (a.ins + 511) / 512;
    a.tiles = (a.outs + 16 * R - 1) / (16 * R);
    // One workgroup a CU, so that x is laid out there once.  A tile a workgroup (several where there are more tiles than that), the other
    // waves share its inner index.
    int groups = 0;
    bool whole = false;
    auto cut = [&](int slices) {                             // the launch with so many slices; us that depend on their number
        a.slice = (a.quads + slices - 1) / slices;
        a.slices = (a.quads + a.slice - 1) / a.slice;
        whole = a.slice * (int64_t)quad + SUMS <= MATVEC_LDS;
        a.chunk = whole ? a.slice : MATVEC_LDS / quad < a.slice - 1 ? MATVEC_LDS / quad : a.slice - 1;
        a.chunk = a.chunk < 1 ? 1 : a.chunk;
        int wgs = ctx->n_cu / (gy * a.slices);
        wgs = a.slices == 1 && wgs < 16 ? 16 : wgs;          // many groups of rows: few workgroups more than CUs would leave most of them idle at the end
        const int each = (a.tiles + wgs - 1) / wgs;
        a.tw = 1;
        while (a.tw < each && a.tw < WAVES) a.tw *= 2;
        a.ks = 1;
        while (a.ks * a.tw < WAVES && a.ks < a.chunk) a.ks *= 2;
        groups = (a.tiles + a.tw - 1) / a.tw;
        groups = groups < wgs ? groups : wgs;
        const int rounds = (a.tiles + groups * a.tw - 1) / (groups * a.tw), full = a.slice / a.chunk, rest = a.slice % a.chunk;
        const int depth = rounds * (full * ((a.chunk + a.ks - 1) / a.ks) + (rest + a.ks - 1) / a.ks);          // stretches a wave goes through
        const float laid = (float)(K::PARTS * 512 * 2) * M * a.slice * (whole ? 1 : rounds), read = (float)rounds * a.tw * R * 16 * 272 * a.slice;
        const float join = a.slices == 1 ? 0.f : (a.slices > 8 ? 3.9f : 2.9f) + 1.1e-6f * a.slices * gy * a.tiles * (R * MT * 1024.f);
        return 25e-6f * laid + 14e-6f * read + 1.7f * depth + join;
    };
    // The inner index may be cut into slices too, a workgroup each, whose sums are joined in the same launch: where x is long, or the tiles are
    // few, a workgroup's slice of x takes less than the whole of it.  A line through times of 72 shapes (1 to 64 rows, 64 to 4096 outputs, 1024 to
    // 16384 inputs, fp32 and bf16 rows and 8-bit ones on a product since taken out) at nine numbers of slices, 10 % off in the mean, tells when: 25 us a MB of x laid out in LDS, 14 a MB of weights
    // that a workgroup reads, 1.7 a stretch that a wave goes through one after another, 2.9 for the join, 1 more for a second batch of loads there, 1.1 a MB
    // of sums.  What it picks is 1 % slower than the best of the nine in the mean, 11 % at most.  fp32 rows, 16 x 256 x 16384: 64.6 us as a
    // whole, 12.9 in 16 slices; 1 x 4096 x 1024 5.6 and 8.3 in two.
    int best = 1;
    if (a.quads > 1) {
        float least = cut(1);
        for (int slices : {2, 4, 6, 8, 11, 16, 22, 32}) {
            if (slices > a.quads || gy * slices > ctx->n_cu || (size_t)slices * gy * a.tiles * (R * MT * 1024) > (size_t)SEQ_ROWS(ctx) * SEQ_ROW_BYTES(RH_SEQ_MAX_DIM)) break;
            const float us = cut(slices);
            if (us < least) { least = us; best = slices; }
        }
    }
    cut(best);
    // waves, and as many more as have pieces of x to lay out, four a thread; two of fp32 rows, which are cut (16 x 1024 x 510: eight 7.7 us, four 6.5,
    // two 5.7; bf16 rows, 16 x 1024 x 512, 4.4, 4.3, 4.6, 64 x 1024 x 510 6.1, 5.5, 5.5)
    constexpr int SHARE = 64 * (XT == RH_T_F32 ? 2 : 4);
    const int64_t pieces = (int64_t)a.chunk * (512 / MATVEC_PIECE) * M;
    int waves = a.tw * a.ks;
    while (waves < WAVES && (int64_t)waves * SHARE <= pieces) ++waves;
    a.threads = 64 * waves;
    const dim3 grid(groups, gy, a.slices), block(a.threads);
    const size_t lds = whole ? (size_t)a.slice * quad + (a.ks > 1 ? SUMS : 0) : MATVEC_LDS;
    auto launch = [&](auto split, auto ends) {
        hipLaunchKernelGGL((k_seq_matvec<XT, MT, R, decltype(split)::value != 0, decltype(ends)::value != 0>), grid, block, lds, ctx->stream, a);
    };
    const bool ends = a.ins % 512 != 0;
    if (a.slices > 1) { if (ends) launch(seq_const<1>(), seq_const<1>()); else launch(seq_const<1>(), seq_const<0>()); }
    else if (ends) launch(seq_const<0>(), seq_const<1>());
    else launch(seq_const<0>(), seq_const<0>());
    return hipGetLastError();
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
    matvec_args a = {};
    a.x = x; a.x_scale = x_scale; a.w = w; a.w_scale = w_scale; a.y = y; a.x_stride = x_stride; a.y_stride = y_stride;
    a.rows = n_rows; a.outs = n_out; a.ins = n_in; a.blocks = (n_in + 31) / 32; a.relu = relu; a.y_f32 = y_type == RH_T_F32;
    rh_status ws = seq_counters(ctx);
    if (ws == RH_OK) ws = seq_scratch(ctx);
    if (ws != RH_OK) return ws;
    a.part = (uint64_t*)ctx->seq_ws; a.count = ctx->seq_cnt;
    // Rows a pass: more read the weights fewer times; what x takes of the LDS, and sums of registers, bounds them.
    hipError_t e;
    if (x_type == RH_T_F32) e = launch_matvec<RH_T_F32, 1, 1>(ctx, a);
    else if (x_type == RH_T_BF16) e = n_rows <= 16 ? launch_matvec<RH_T_BF16, 1, 1>(ctx, a) : launch_matvec<RH_T_BF16, 2, 2>(ctx, a);
    else e = n_rows <= 16 ? launch_matvec<RH_T_E4M3, 1, 1>(ctx, a) : launch_matvec<RH_T_E4M3, 2, 2>(ctx, a);
    RH_HIP(ctx, e);
    return RH_OK;
}
