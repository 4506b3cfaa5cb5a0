// rh_cache_attend: attention of one new token of every stream over a paged cache.
//
// Bound by memory: every key and value of a stream is read once for all query heads that share it.  The scores and the sums go on the
// matrix cores, which have rate to spare even where a tile of 16 heads is mostly empty (64 streams of up to 8192 tokens, bf16, 32 heads
// on 8 of 128: 204 us, 5.2 TB/s, as much as a copy has; they work 7 % of the time), so that one kernel serves every number of heads a key,
// and vector instructions are left for the softmax.
//
// A wave takes a tile of tokens (32; 16 of an fp32 cache) at a time, with no barrier in its loop:
//   scores   S^T[token][head] = K Q^T: the keys are the matrix operand, 8 (4) elements of a token a lane
//   softmax  one lane has the scores of one head, so the running maximum, the sums and the factors stay in the lane; only the
//            maximum over a tile crosses lanes (two exchanges)
//   sums     O^T[d][head] += V^T P^T: the weights are in the lanes that the product wants them in when its inner index runs over
//            the tokens in the order of the scores' registers; a lane loads E consecutive elements of each of its tokens, and the
//            product's rows are taken as d = E*m + e for the E products of that load, so that a transposition inside the lane (a byte
//            permutation for two 16-bit values, none for fp32) is all that the values need
// A weight goes into the 16-bit product as the sum of three bf16 numbers, which together are the weight exactly; they have its sign, so that an infinite
// value gives the infinity that the weight gives, and not the NaN of two infinities.  An e4m3 key's scale multiplies its score, a value's scale its weight.
//
// Work is split over the streams' lengths: all streams' tiles (times the head units) are cut into chunks of equal size, so that a long stream
// among short ones keeps every CU busy.  How long a chunk is follows from the lengths, which the host does not know: every
// wave (of more than 64 streams, every workgroup) adds them up and finds its own chunk.  The chunks of a stream and unit leave their
// sums, maxima and totals in scratch memory; of every 16 the one that finishes last joins them, in their order, and so on up.  One stream
// of 108000 tokens (e4m3, 16 heads on 2 of 128: 242 chunks, two levels): 24.7 us, where its bytes take 10.9; 5 are a call's on one tile,
// about 3 each level, and the four waves a CU that this gives keep too few bytes in flight.
#include "seq_common.h"

struct attend_args {
    const void *k, *v, *q;
    const float *k_scale, *v_scale;
    int64_t ks[3], vs[3], qs[2];
    const int32_t *table, *lengths;
    void* out;
    float *lse, *ws;
    uint32_t* count;
    seq_div page;
    int32_t n_pages, heads, q_heads, group, head_tiles, max_pages, n_streams, window, n_cu, grouped;
    float scale;             // times log2(e): the softmax runs on powers of two
};

#define ATTEND_WAVES 4
#define ATTEND_T (64 * ATTEND_WAVES)
#define ATTEND_CHUNK_MIN 4       // tiles
#define ATTEND_WHOLE 8           // tiles, where no stream has more
#define ATTEND_CHUNK_FEW 32      // tiles a chunk up to which each CU gets one chunk; beyond, ATTEND_CHUNKS
#define ATTEND_SOLO 8            // tiles of a stream that a wave takes alone, where there are many such streams and none longer
#define ATTEND_GROUPED 64        // chunks of all streams from which on a chunk's units go to one XCD
#define ATTEND_FAN 16            // chunks joined at a time, at most

template <int KIND> struct attend_kind;
template <> struct attend_kind<RH_T_F32> { typedef float Q; typedef float C; static constexpr int TT = 1; };
template <> struct attend_kind<RH_T_BF16> { typedef __bf16 Q; typedef __bf16 C; static constexpr int TT = 2; };
template <> struct attend_kind<RH_T_E4M3> { typedef __bf16 Q; typedef uint8_t C; static constexpr int TT = 2; };

template <int N> struct attend_words { uint32_t w[N]; };
template <int N> __device__ __forceinline__ void attend_get(uint32_t* to, const void* from)
{
    static_assert(N == 1 || N == 2 || N == 4, "");
    if constexpr (N == 1) to[0] = *(const uint32_t*)from;
    else if constexpr (N == 2) { const uint2 u = *(const uint2*)from; to[0] = u.x; to[1] = u.y; }
    else { const uint4 u = *(const uint4*)from; to[0] = u.x; to[1] = u.y; to[2] = u.z; to[3] = u.w; }
}
// bytes of LDS for the keys and for the sums, whichever is more
template <int KIND, int D> constexpr int attend_lds()
{
    constexpr int keys = ATTEND_WAVES * 16 * attend_kind<KIND>::TT * (D * (int)sizeof(typename attend_kind<KIND>::C) + 16);
    constexpr int sums = ATTEND_WAVES / 2 * (D / 16 + 1) * 64 * (int)sizeof(f32x4);
    return keys > sums ? keys : sums;
}

// MANY: more than 64 streams
template <int KIND, int D, bool MANY>
__global__ __launch_bounds__(ATTEND_T, D <= 128 ? 2 : 1) void k_seq_attend(attend_args a)
{
    typedef typename attend_kind<KIND>::Q Q;
    typedef typename attend_kind<KIND>::C C;
    constexpr int TT = attend_kind<KIND>::TT, TILE = 16 * TT, ROWS = 4 * TT;       // token tiles of 16, tokens, values' rows a lane
    constexpr int KW = KIND == RH_T_F32 ? D / 4 : D / 8;                           // words of Q (fp32 or bf16) a lane
    constexpr int RB = D * sizeof(C), PITCH = RB + 16;                             // bytes of a key, and of its row in LDS (an odd number of 16: no conflicts)
    constexpr int LPR = RB / 16, NK = TILE * LPR / 64;                             // lanes a key, loads a lane and tile
    constexpr int VL = (D / 16 * sizeof(C) + 3) / 4;                               // words of V a lane and token (e4m3: the last may be half a word)
    constexpr int NT = D / 16;                                                     // products' row tiles
    // V: lane c has E consecutive elements of each stretch of 16*E: those of 16 bytes (8 of e4m3) first, then what is left
    constexpr int EM = KIND == RH_T_F32 ? 4 : 8, NB = D / (16 * EM), HAS4 = EM == 8 && D % 128 >= 64, HAS2 = D % 64 >= 32;

    extern __shared__ uint4 s_mem[];                         // the waves' keys; behind the loop, what half of the waves hand to the others
    f32x4(*s_acc)[NT + 1][64] = (f32x4(*)[NT + 1][64])s_mem;
    __shared__ float s_some[ATTEND_WAVES];
    __shared__ int32_t s_most[ATTEND_WAVES], s_sums[2][ATTEND_WAVES];
    __shared__ uint32_t s_last;

    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, c = lane & 15, j = lane >> 4;
    const int units = a.heads * a.head_tiles;

    // ---- the streams' chunks: streams in order, each cut into chunks of `chunk` tiles.  Up to 64 streams every wave has one a lane;
    // of more, a thread has `per` neighbours, and running sums go to LDS.
    constexpr int PER = MANY ? RH_SEQ_MAX_STREAMS / ATTEND_T : 1;
    const int per = MANY ? (a.n_streams + ATTEND_T - 1) / ATTEND_T : 1, b0 = MANY ? t * per : lane;
    int32_t* s_first = (int32_t*)((uint8_t*)s_mem + attend_lds<KIND, D>());       // chunks before a stream, and of those before it the ones that need scratch memory
    int32_t* s_row = s_first + RH_SEQ_MAX_STREAMS + 1;
    const int64_t row_cap = (int64_t)a.max_pages * a.page.d;
    auto clipped = [&](int b) -> int32_t { const int32_t n = a.lengths[b]; return n < 0 ? 0 : n > row_cap ? (int32_t)row_cap : n; };
    auto tiles_of = [&](int32_t len) -> int32_t {
        const uint32_t n = a.window && len > a.window ? a.window : len;
        return (int32_t)((n + TILE - 1) / TILE);
    };
    int32_t len[PER] = {}, most_tiles = 0;                   // unused beyond `per`
    float some = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per) break;
        len[i] = b0 + i < a.n_streams ? clipped(b0 + i) : 0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per) break;
        const int32_t n = tiles_of(len[i]);
        some += (float)n;
        most_tiles = n > most_tiles ? n : most_tiles;
    }
    // Many short streams: a wave each, with nothing to join.  (128 streams of up to 256 tokens, 8 heads: 24.0 -> 19.5 us, of up to 64
    // 16.7 -> 10.0.  Half as many streams gain up to fewer tiles: 64 of up to 30 tokens 7.1 -> 6.0, of up to 128 10.7 -> 12.2.)
    const int few = a.n_streams * units / a.n_cu, cap = few < 4 ? few / 2 : ATTEND_SOLO;
    bool longer = __any(most_tiles > cap), several = __any(most_tiles > ATTEND_WHOLE);
    some = seq_sum(some);
    if constexpr (MANY) {
        if (lane == 0) { s_some[wave] = some; s_most[wave] = longer + 2 * several; }
        __syncthreads();
        some = 0.f; longer = several = false;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) { some += s_some[w]; longer |= s_most[w] & 1; several |= s_most[w] >> 1; }
    }
    const bool solo = !longer;
    const float all = some * (float)units, cus = (float)a.n_cu;
    // at most 2^30, which no stream has (a length is below 2^31, a tile 16 or more): the sums' rounding and their size are both covered
    int chunk = (int)fminf(ceilf(fmaxf(fminf(all / cus, (float)ATTEND_CHUNK_FEW), all / (cus * ATTEND_CHUNKS) * 1.0001f)), 0x1p30f);
    // Two tiles a wave take less than a join where no stream has more (8 streams of up to 200 tokens, bf16, 2 heads of 128 8.9 -> 8.2 us; with
    // streams of 300 among them 9.1 -> 10.5; fp32, 8 heads of 64, 100 tokens 7.7 -> 6.9, of 192, 93 tokens 11.5 -> 12.1: tiles of long rows take longer)
    const int least = !several && RB <= 512 ? ATTEND_WHOLE : ATTEND_CHUNK_MIN;
    chunk = solo ? ATTEND_SOLO : ((chunk < least ? least : chunk) + ATTEND_WAVES - 1) / ATTEND_WAVES * ATTEND_WAVES;
    // a stream without tokens has one chunk, which writes its zeros; only chunks of streams that have several need scratch memory
    int32_t n_chunks[PER], mine = 0, shared = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per) break;
        const int32_t n = tiles_of(len[i]);
        n_chunks[i] = b0 + i >= a.n_streams ? 0 : 1;
        if (n > chunk) n_chunks[i] = (n + chunk - 1) / chunk;
        mine += n_chunks[i];
        shared += n_chunks[i] > 1 ? n_chunks[i] : 0;
    }
    int32_t before = seq_scan(mine), ahead = seq_scan(shared), pairs = __builtin_amdgcn_readlane(before, 63);
    before -= mine; ahead -= shared;
    if constexpr (MANY) {
        if (lane == 63) { s_sums[0][wave] = before + mine; s_sums[1][wave] = ahead + shared; }
        __syncthreads();
        pairs = 0;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) {
            if (w < wave) { before += s_sums[0][w]; ahead += s_sums[1][w]; }
            pairs += s_sums[0][w];
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i >= per) break;
            if (b0 + i < a.n_streams) { s_first[b0 + i] = before; s_row[b0 + i] = ahead; }
            before += n_chunks[i]; ahead += n_chunks[i] > 1 ? n_chunks[i] : 0;
        }
        if (t == 0) s_first[a.n_streams] = pairs;
        __syncthreads();
    }

    // ---- this wave's chunk
    // Workgroups are dealt out to the eight XCDs in turn.  Where the units of a chunk read lines in common - a second tile of heads all of
    // them, cache heads that lie side by side in parts of a line those - they go to the same XCD, whose L2 then has them (16 streams
    // of up to 8000 tokens, 8 x 20 heads 89 -> 77 us; up to 32000 of e4m3, 8 x 4 heads of 64 94 -> 74).  Elsewhere, or with few
    // chunks, that would only load the XCDs less evenly (8 x 1 heads of 128 58 -> 62).
    int pair, unit;
    if (solo || !a.grouped || pairs < ATTEND_GROUPED) {
        const int64_t index = solo ? (int64_t)blockIdx.x * ATTEND_WAVES + wave : (int64_t)blockIdx.x;
        if (index >= (int64_t)pairs * units) return;         // the grid is as large as any lengths need; a workgroup's waves part only where they go alone
        pair = (int)((uint32_t)index / (uint32_t)units); unit = (int)((uint32_t)index % (uint32_t)units);
    } else {
        const uint32_t k = blockIdx.x >> 3;
        pair = (int)(k / (uint32_t)units * 8 + (blockIdx.x & 7)); unit = (int)(k % (uint32_t)units);
        if (pair >= pairs) return;
    }
    int b = 0, length, split, n_split, first_row;
    if constexpr (MANY) {
        for (int hi = a.n_streams; hi - b > 1;) { const int mid = (b + hi) >> 1; if (s_first[mid] <= pair) b = mid; else hi = mid; }
        b = __builtin_amdgcn_readfirstlane(b);
        const int first = __builtin_amdgcn_readfirstlane(s_first[b]);
        split = pair - first; n_split = __builtin_amdgcn_readfirstlane(s_first[b + 1]) - first;
        first_row = __builtin_amdgcn_readfirstlane(s_row[b]);
        length = clipped(b);
    } else {
        b = __builtin_ctzll(__ballot(pair >= before && pair < before + mine));
        length = __builtin_amdgcn_readlane(len[0], b); split = pair - __builtin_amdgcn_readlane(before, b);
        n_split = __builtin_amdgcn_readlane(mine, b); first_row = __builtin_amdgcn_readlane(ahead, b);
    }
    const int32_t n_kept = a.window && length > a.window ? a.window : length, begin = length - n_kept;
    const int32_t n_tiles = (int32_t)(((int64_t)n_kept + TILE - 1) / TILE);
    const int32_t tile_end = n_tiles < (split + 1) * chunk ? n_tiles : (split + 1) * chunk;

    const int kvh = unit / a.head_tiles, h0 = kvh * a.group + unit % a.head_tiles * 16;
    const int ng = (kvh + 1) * a.group - h0 < 16 ? (kvh + 1) * a.group - h0 : 16;

    // ---- queries: lane (head c, quarter j); heads that are none are zeros
    uint32_t q[KW];
    {
        const Q* qp = (const Q*)a.q + b * a.qs[0] + (h0 + (c < ng ? c : 0)) * a.qs[1];
#pragma unroll
        for (int s = 0; s < KW / 4; ++s) {
            // the elements that the keys' loads give this quarter
            int d;
            if constexpr (KIND == RH_T_F32) d = 16 * s + 4 * j;
            else if constexpr (KIND == RH_T_BF16) d = 32 * s + 8 * j;
            else d = s < D / 64 * 2 ? 64 * (s / 2) + 16 * j + 8 * (s & 1) : D / 64 * 64 + 8 * j;
            const uint4 u = seq_load<uint4>(qp + d);
            q[4 * s] = c < ng ? u.x : 0; q[4 * s + 1] = c < ng ? u.y : 0; q[4 * s + 2] = c < ng ? u.z : 0; q[4 * s + 3] = c < ng ? u.w : 0;
        }
    }

    // ---- the tokens of a tile: lane l looks after token l % TILE
    struct where { int64_t k, v; float ks, vs; bool ok; };
    const int32_t* table = a.table + (int64_t)b * a.max_pages;
    auto entry = [&](int32_t tile) -> int32_t {              // the table's word for this lane's token, -1 behind the last
        const uint32_t pos = (uint32_t)begin + (uint32_t)tile * TILE + (lane & (TILE - 1));
        const bool in = tile < tile_end && pos < (uint32_t)length;
        const int32_t p = table[in ? seq_quot(pos, a.page) : 0];         // no branch around the load: the loads in flight stay countable
        return in ? p : -1;
    };
    auto place = [&](int32_t tile, int32_t p) -> where {
        const uint32_t pos = (uint32_t)begin + (uint32_t)tile * TILE + (lane & (TILE - 1));
        const uint32_t line = pos - seq_quot(pos, a.page) * a.page.d;
        where w;
        w.ok = p >= 0 && p < a.n_pages;
        const int64_t pp = w.ok ? p : 0, ll = w.ok ? line : 0;   // what is left out reads page 0's first line, and counts for nothing
        w.k = pp * a.ks[0] + ll * a.ks[1];
        w.v = pp * a.vs[0] + ll * a.vs[1];
        if constexpr (KIND == RH_T_E4M3) {
            const int64_t at = (pp * a.heads + kvh) * a.page.d + ll;
            w.ks = a.k_scale[at]; w.vs = a.v_scale[at];
        } else w.ks = w.vs = 1.f;
        return w;
    };
    auto from = [](int64_t v, int l) -> int64_t {
        const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)v, l), hi = (uint32_t)__shfl((int)(v >> 32), l);
        return (int64_t)((uint64_t)hi << 32 | lo);
    };
    const C* kbase = (const C*)a.k + kvh * a.ks[2];
    const C* vbase = (const C*)a.v + kvh * a.vs[2];
    // Keys come in whole: consecutive lanes take consecutive 16 bytes, so that a line is asked for once, and pass through LDS to the
    // lanes that the products want them in.  (Loaded there at once, a quarter wave touches 16 lines, and each of them again: 64 x 8192
    // tokens of bf16 215.5 -> 218.3 us, 108000 of e4m3 43.1 -> 46.4.)
    uint8_t* keys = (uint8_t*)s_mem + wave * TILE * PITCH;
    u32x4 kr[NK];
    uint32_t vr[ROWS][VL];
    auto load_k = [&](const where& w) {
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            const int tok = (64 * n + lane) / LPR, piece = (64 * n + lane) % LPR;
            kr[n] = *(const u32x4*)((const uint8_t*)(kbase + from(w.k, tok)) + 16 * piece);
        }
    };
    auto stage_k = [&]() {
#pragma unroll
        for (int n = 0; n < NK; ++n) *(u32x4*)(keys + (64 * n + lane) / LPR * PITCH + (64 * n + lane) % LPR * 16) = kr[n];
    };
    auto load_v = [&](const where& w) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const C* p = vbase + from(w.v, 16 * (r >> 2) + 4 * j + (r & 3));
            constexpr int WM = EM * sizeof(C) / 4;           // words of a stretch's lane
#pragma unroll
            for (int s = 0; s < NB; ++s) attend_get<WM>(&vr[r][WM * s], p + 16 * EM * s + EM * c);
            if constexpr (HAS4) attend_get<WM / 2>(&vr[r][WM * NB], p + 128 * NB + 4 * c);
            if constexpr (HAS2) {
                constexpr int at = WM * NB + (HAS4 ? WM / 2 : 0), d0 = 16 * EM * NB + (HAS4 ? 64 : 0);
                if constexpr (KIND == RH_T_E4M3) vr[r][at] = *(const uint16_t*)(p + d0 + 2 * c);
                else attend_get<sizeof(C) / 2>(&vr[r][at], p + d0 + 2 * c);
            }
        }
    };

    f32x4 acc[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, total = 0.f;

    const int turn = solo ? 1 : ATTEND_WAVES;                // tiles from one of a wave's to its next
    int32_t tile = split * chunk + (solo ? 0 : wave);
    if (tile < tile_end) {
        where now = place(tile, entry(tile));
        load_k(now);
        load_v(now);
        int32_t next_entry = entry(tile + turn);
        auto step = [&](auto has_next) __attribute__((always_inline)) {
            constexpr bool MORE = decltype(has_next)::value != 0;
            // scores: rows 4*j + i of token tile tt, head c
            stage_k();
            f32x4 sc[TT];
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                sc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
                const uint8_t* key = keys + (16 * tt + c) * PITCH;
                auto product = [&](attend_words<4> ka, int s) {
                    attend_words<4> qa;
#pragma unroll
                    for (int w = 0; w < 4; ++w) qa.w[w] = q[4 * s + w];
                    sc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ka), __builtin_bit_cast(bf16x8, qa), sc[tt], 0, 0, 0);
                };
                auto wide = [](uint32_t x, uint32_t y) {
                    return attend_words<4>{seq_e4m3_pair<false>(x), seq_e4m3_pair<true>(x), seq_e4m3_pair<false>(y), seq_e4m3_pair<true>(y)};
                };
#pragma unroll
                for (int s = 0; s < RB / 64; ++s) {
                    const uint4 u = *(const uint4*)(key + 64 * s + 16 * j);
                    if constexpr (KIND == RH_T_F32) {
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            sc[tt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), __uint_as_float(q[4 * s + e]), sc[tt], 0, 0, 0);
                    } else if constexpr (KIND == RH_T_BF16) product(attend_words<4>{u.x, u.y, u.z, u.w}, s);
                    else { product(wide(u.x, u.y), 2 * s); product(wide(u.z, u.w), 2 * s + 1); }
                }
                if constexpr (RB % 64) {
                    const uint2 u = *(const uint2*)(key + RB / 64 * 64 + 8 * j);
                    product(wide(u.x, u.y), RB / 64 * 2);
                }
            }
            // the next tile's keys, into the registers that the products have read
            where next;
            int32_t after;
            if constexpr (MORE) {
                next = place(tile + turn, next_entry);
                load_k(next);
                after = entry(tile + 2 * turn);
            }

            // softmax over this tile: token 16*tt + 4*j + i is lane (16*tt + 4*j + i)'s
            float p[ROWS], vs[ROWS], most = -INFINITY;
            const uint64_t oks = __ballot(now.ok);
            const bool whole = oks == ~0ull;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int tok = 16 * (r >> 2) + 4 * j + (r & 3);
                float s = sc[r >> 2][r & 3];
                if constexpr (KIND == RH_T_E4M3) { s *= __shfl(now.ks, tok); vs[r] = __shfl(now.vs, tok); }
                s *= a.scale;
                if (!whole) s = oks >> tok & 1 ? s : -INFINITY;
                p[r] = s;
                most = fmaxf(most, s);
            }
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const float up = fmaxf(top, most), base = up == -INFINITY ? 0.f : up;
            const float fade = __builtin_amdgcn_exp2f(top - base);
            top = up;
            float part = 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) { p[r] = __builtin_amdgcn_exp2f(p[r] - base); part += p[r]; }
            total = total * fade + part;
            if (!__all(fade == 1.f)) {
#pragma unroll
                for (int i = 0; i < NT; ++i) acc[i] *= fade;
            }
            // tokens that are left out have weight zero: their values must not be infinite or NaN
            if (!whole) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const bool ok = oks >> (16 * (r >> 2) + 4 * j + (r & 3)) & 1;
#pragma unroll
                    for (int w = 0; w < VL; ++w) vr[r][w] = ok ? vr[r][w] : 0;
                    if constexpr (KIND == RH_T_E4M3) vs[r] = ok ? vs[r] : 0.f;
                }
            }
            // sums
            if constexpr (KIND == RH_T_F32) {
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[r][i]), p[r], acc[i], 0, 0, 0);
            } else {
                attend_words<4> part[3];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t cut[2][3];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x = p[2 * w + h];
                        if constexpr (KIND == RH_T_E4M3) x *= vs[2 * w + h];
                        auto first = [](float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); };      // its eight leading bits
                        const float hi = first(x);
                        float r = x - hi;
                        if constexpr (KIND == RH_T_E4M3) r = x == hi ? 0.f : r;           // an infinite scale; the values are finite
                        // no part of a weight above zero is zero, or an infinite value would make it NaN
                        else r = fmaxf(r, hi * 0x1p-30f);
                        const float mid = first(r);
                        float lo = r - mid;
                        if constexpr (KIND == RH_T_BF16) lo = fmaxf(lo, hi * 0x1p-30f);
                        cut[h][0] = __float_as_uint(hi); cut[h][1] = __float_as_uint(mid); cut[h][2] = __float_as_uint(lo);
                    }
#pragma unroll
                    for (int k = 0; k < 3; ++k) part[k].w[w] = __builtin_amdgcn_perm(cut[1][k], cut[0][k], 0x07060302u);
                }
#pragma unroll
                for (int i = 0; i < NT; i += 2) {
                    attend_words<4> even, odd;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t x, y;
                        if constexpr (KIND == RH_T_BF16) { x = vr[2 * w][i / 2]; y = vr[2 * w + 1][i / 2]; }
                        else {
                            x = i & 2 ? seq_e4m3_pair<true>(vr[2 * w][i / 4]) : seq_e4m3_pair<false>(vr[2 * w][i / 4]);
                            y = i & 2 ? seq_e4m3_pair<true>(vr[2 * w + 1][i / 4]) : seq_e4m3_pair<false>(vr[2 * w + 1][i / 4]);
                        }
                        even.w[w] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                        odd.w[w] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                    }
                    const bf16x8 va = __builtin_bit_cast(bf16x8, even), vb = __builtin_bit_cast(bf16x8, odd);
#pragma unroll
                    for (int k = 2; k >= 0; --k) {
                        const bf16x8 pw = __builtin_bit_cast(bf16x8, part[k]);
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pw, acc[i], 0, 0, 0);
                        acc[i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, pw, acc[i + 1], 0, 0, 0);
                    }
                }
            }
            if constexpr (MORE) {
                load_v(next);
                now = next;
                next_entry = after;
            }
        };
        for (; tile + turn < tile_end; tile += turn) step(seq_const<1>());
        step(seq_const<0>());
    }

    // ---- joining: one set of sums, maximum and total (of this lane's tokens) with another of the same lane
    auto join = [&](auto other) __attribute__((always_inline)) {
        const f32x4 stat = other(NT);
        const float up = fmaxf(top, stat[0]), base = up == -INFINITY ? 0.f : up;
        const float f = __builtin_amdgcn_exp2f(top - base), g = __builtin_amdgcn_exp2f(stat[0] - base);
        top = up;
        total = total * f + stat[1] * g;
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i] = acc[i] * f + other(i) * g;
    };
    const int busy = solo ? 1 : tile_end - split * chunk;    // tiles of the chunk, and so waves that had any
    auto join_waves = [&]() __attribute__((always_inline)) {               // into wave 0
#pragma unroll
        for (int n = ATTEND_WAVES / 2; n; n >>= 1) {
            if (n >= busy) continue;
            // wave 1 hands over where only it has read
            if (wave >= n && wave < 2 * n) {
                f32x4(*o)[64] = s_acc[n == 1 ? 1 : wave - n];
#pragma unroll
                for (int i = 0; i < NT; ++i) o[i][lane] = acc[i];
                o[NT][lane] = f32x4{top, total, 0.f, 0.f};
            }
            __syncthreads();
            if (wave < n) {
                f32x4(*o)[64] = s_acc[n == 1 ? 1 : wave];
                join([&](int i) { return o[i][lane]; });
            }
        }
    };
    auto write = [&]() __attribute__((always_inline)) {                    // wave 0: the outputs
        if (c >= ng) return;
        const int64_t row = (int64_t)b * a.q_heads + h0 + c;
        // a NaN total has to show; a total of zero is a stream without tokens
        const float f = total > 0.f ? 1.f / total : total != total ? total : 0.f;
        if (j == 0 && a.lse) a.lse[row] = total > 0.f ? (top + __builtin_amdgcn_logf(total)) * 0.69314718056f : total != total ? total : -INFINITY;
        Q* out = (Q*)a.out + row * D;
        // the products of a stretch that starts at element d0 hold d = d0 + E*(4*j + r) + e
#pragma unroll
        for (int i = 0; i < NT;) {
            const int E = i < EM * NB ? EM : HAS4 && i < 8 * NB + 4 ? 4 : 2;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                Q* o = out + 16 * i + E * (4 * j + r);
                if constexpr (sizeof(Q) == 4) {
                    if (E == 2) *(float2*)o = make_float2(acc[i][r] * f, acc[i + 1][r] * f);
#pragma unroll
                    for (int e = 0; e + 3 < E; e += 4)
                        *(f32x4*)(o + e) = f32x4{acc[i + e][r] * f, acc[i + e + 1][r] * f, acc[i + e + 2][r] * f, acc[i + e + 3][r] * f};
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < E; e += 2) w[e / 2] = seq_pack_bf16(acc[i + e][r] * f, acc[i + e + 1][r] * f);
                    if (E == 8) *(uint4*)o = make_uint4(w[0], w[1], w[2], w[3]);
                    else if (E == 4) *(uint2*)o = make_uint2(w[0], w[1]);
                    else *(uint32_t*)o = w[0];
                }
            }
            i += E;
        }
    };

    if (busy > 1) {
        __syncthreads();                                     // no wave needs its keys any more
        join_waves();
    }
    if (wave == 0 || solo) {
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
    }
    // ---- several chunks: sums to scratch memory, rows of [tile][quarter][head]; of every ATTEND_FAN the one that comes last joins them.
    // The chunks of a stream sit on eight XCDs with an L2 each: what they leave is stored through (relaxed atomics of the device's scope) and
    // loaded past the L2, and a wave's stores are acknowledged before the chunk is counted.  (Fences, which write the whole L2 back, took
    // 490 of 690 us on 64 x 8192 tokens.)
    struct two { uint64_t u[2]; };
    constexpr int ROW = SEQ_ROW_BYTES(D) / 8;                // words of a row
    const size_t step = (size_t)units * ROW;
    uint64_t* rows = (uint64_t*)a.ws + ((size_t)first_row * units + unit) * ROW;
    uint32_t* counts = a.count + (size_t)first_row * units + unit;
    int at = split, members = n_split, stride = 1;           // the row that this workgroup has made, as the at-th of `members`, `stride` rows apart
    // two levels of about as many each, where one does not do.  Groups of 16 and of 12, us, one stream, 16 heads on 2 of 128 in bf16: 17 chunks 12.3 and 11.8, 48 12.4 and
    // 11.9, 64 12.8 and 13.5, 96 14.7 and 14.4, 128 15.7 and 15.3; e4m3 12.1 and 11.6 (17), 13.8 and 13.5 (128); dim 256 18.7 and 17.6, 24.2 and 23.3; fp32 of 64 9.3
    // and 9.3, 10.5 and 10.7
    const int fan = n_split > ATTEND_FAN && n_split <= 144 ? 12 : ATTEND_FAN;
    for (int level = 0; members > 1; ++level) {
        const int first = at / fan * fan, n = members - first < fan ? members - first : fan;
        if (n > 1) {
            if (wave == 0) {
                uint64_t* o = rows + (size_t)at * stride * step;
                if (c < ng) {
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const two w = __builtin_bit_cast(two, acc[i]);
                        uint64_t* p = o + ((4 * i + j) * ng + c) * 2;
                        __hip_atomic_store(p, w.u[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        __hip_atomic_store(p + 1, w.u[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                    if (j == 0)
                        __hip_atomic_store(o + NT * 128 + c, (uint64_t)__float_as_uint(total) << 32 | __float_as_uint(top), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (lane == 0) {
                    // a group of a higher level holds more than fan rows: a counter of its own beside the lower levels'
                    uint32_t* count = counts + (size_t)(first * stride + level) * units;
                    const bool last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)n - 1;
                    if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    s_last = last;
                }
            }
            __syncthreads();
            if (!s_last) return;
            // all rows of the group at once: one thread a vector of sums
            const uint64_t* o = rows + (size_t)first * stride * step;
            auto join_rows = [&](auto most) __attribute__((always_inline)) {
                constexpr int N = decltype(most)::value;
                for (int x = t; x < NT * 4 * ng; x += ATTEND_T) {
                    const int h = x % ng, quarter = x / ng;
                    uint64_t stat[N];
                    two v[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const uint64_t* p = o + (size_t)(k < n ? k : 0) * stride * step;
                        stat[k] = __hip_atomic_load(p + NT * 128 + h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        v[k].u[0] = __hip_atomic_load(p + x * 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        v[k].u[1] = __hip_atomic_load(p + x * 2 + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                    float m = -INFINITY, tot = 0.f;
#pragma unroll
                    for (int k = 0; k < N; ++k) if (k < n) m = fmaxf(m, __uint_as_float((uint32_t)stat[k]));
                    const float base = m == -INFINITY ? 0.f : m;
                    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        if (k >= n) continue;
                        const float f = __builtin_amdgcn_exp2f(__uint_as_float((uint32_t)stat[k]) - base);
                        tot += __uint_as_float((uint32_t)(stat[k] >> 32)) * f;
                        sum += __builtin_bit_cast(f32x4, v[k]) * f;
                    }
                    s_acc[0][quarter >> 2][(quarter & 3) * 16 + h] = sum;
                    if (quarter < 4) s_acc[0][NT][quarter * 16 + h] = f32x4{m, tot, 0.f, 0.f};
                }
            };
            if (n <= 4) join_rows(seq_const<4>()); else if (n <= 12) join_rows(seq_const<12>()); else join_rows(seq_const<ATTEND_FAN>());
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int i = 0; i < NT; ++i) acc[i] = s_acc[0][i][lane];
                const f32x4 stat = s_acc[0][NT][lane];
                top = stat[0]; total = stat[1];
            }
        }
        at /= fan; members = (members + fan - 1) / fan; stride *= fan;
    }
    if (wave == 0 || solo) write();
}

template <int KIND, int D>
static hipError_t launch_attend(rh_ctx* ctx, const attend_args& a, int64_t grid)
{
    constexpr int lds = attend_lds<KIND, D>(), sums = (2 * RH_SEQ_MAX_STREAMS + 1) * (int)sizeof(int32_t);
    static bool attr_done[RH_MAX_DEVICES] = {};              // the attribute is per device
    if (!attr_done[ctx->device]) {
        hipError_t e = hipFuncSetAttribute((const void*)k_seq_attend<KIND, D, false>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e == hipSuccess) e = hipFuncSetAttribute((const void*)k_seq_attend<KIND, D, true>, hipFuncAttributeMaxDynamicSharedMemorySize, lds + sums);
        if (e != hipSuccess) return e;
        attr_done[ctx->device] = true;
    }
    if (a.n_streams > 64) hipLaunchKernelGGL((k_seq_attend<KIND, D, true>), dim3((unsigned)grid), dim3(ATTEND_T), lds + sums, ctx->stream, a);
    else hipLaunchKernelGGL((k_seq_attend<KIND, D, false>), dim3((unsigned)grid), dim3(ATTEND_T), lds, ctx->stream, a);
    return hipGetLastError();
}

template <int KIND>
static hipError_t launch_attend(rh_ctx* ctx, const attend_args& a, int64_t grid, int dim)
{
    switch (dim) {
    case 32: return launch_attend<KIND, 32>(ctx, a, grid);
    case 64: return launch_attend<KIND, 64>(ctx, a, grid);
    case 96: return launch_attend<KIND, 96>(ctx, a, grid);
    case 128: return launch_attend<KIND, 128>(ctx, a, grid);
    case 160: return launch_attend<KIND, 160>(ctx, a, grid);
    case 192: return launch_attend<KIND, 192>(ctx, a, grid);
    case 224: return launch_attend<KIND, 224>(ctx, a, grid);
    default: return launch_attend<KIND, 256>(ctx, a, grid);
    }
}

extern "C" rh_status rh_cache_attend(rh_ctx* ctx, const rh_kv_cache* cache, const void* q, const int64_t q_stride[2], int32_t type,
                                     int32_t q_heads, const int32_t* block_table, int32_t max_pages, const int32_t* lengths,
                                     int32_t n_streams, float scale, int32_t window, void* out, float* lse)
{
    if (!ctx) return RH_E_INVALID;
    if (!cache || !q || !q_stride || !block_table || !lengths || !out) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: null argument");
    if (type != RH_T_F32 && type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: queries of type %d", type);
    const rh_status st = seq_check_cache(ctx, "rh_cache_attend", cache);
    if (st != RH_OK) return st;
    if ((type == RH_T_F32) != (cache->type == RH_T_F32))
        RH_FAIL(ctx, RH_E_UNIMPLEMENTED, "rh_cache_attend: queries of type %d over a cache of type %d", type, cache->type);
    if (q_heads < 1 || q_heads % cache->heads) RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_attend: %d query heads over %d of the cache", q_heads, cache->heads);
    if (n_streams < 1 || n_streams > RH_SEQ_MAX_STREAMS)
        RH_FAIL(ctx, RH_E_CAPACITY, "rh_cache_attend: %d streams outside [1,%d]", n_streams, RH_SEQ_MAX_STREAMS);
    if (max_pages < 1 || (int64_t)max_pages * cache->page > 0x7FFFFFFFll - cache->page)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_attend: %d pages of %d tokens a stream", max_pages, cache->page);
    if ((int64_t)q_heads * n_streams > 0x7FFFFFFFll / RH_SEQ_MAX_DIM) RH_FAIL(ctx, RH_E_SHAPE, "rh_cache_attend: %d heads of %d streams", q_heads, n_streams);
    if (window < 0) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: a window of %d", window);
    if ((uintptr_t)out & 15) RH_FAIL(ctx, RH_E_INVALID, "rh_cache_attend: out must be 16-byte aligned");
    attend_args a;
    a.k = cache->k; a.v = cache->v; a.q = q; a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
    for (int i = 0; i < 3; ++i) { a.ks[i] = cache->k_stride[i]; a.vs[i] = cache->v_stride[i]; }
    for (int i = 0; i < 2; ++i) a.qs[i] = q_stride[i];
    a.table = block_table; a.lengths = lengths; a.out = out; a.lse = lse; a.page = seq_make_div((uint32_t)cache->page);
    a.n_pages = cache->n_pages; a.heads = cache->heads; a.q_heads = q_heads; a.group = q_heads / cache->heads;
    a.head_tiles = (a.group + 15) / 16; a.max_pages = max_pages; a.n_streams = n_streams; a.window = window; a.n_cu = ctx->n_cu;
    a.scale = scale * 1.44269504089f;
    const int64_t size = cache->type == RH_T_F32 ? 4 : cache->type == RH_T_BF16 ? 2 : 1;
    a.grouped = a.head_tiles > 1 || (cache->heads > 1 && (cache->k_stride[2] * size % 128 || cache->v_stride[2] * size % 128));
    // Chunks: at most ATTEND_CHUNKS a CU and one more for every stream and unit; less where the table's rows are short.
    const int64_t units = (int64_t)cache->heads * a.head_tiles, streams_units = units * n_streams;
    const int64_t longest = window && window < (int64_t)max_pages * cache->page ? window : (int64_t)max_pages * cache->page;
    const int tile = cache->type == RH_T_F32 ? 16 : 32;
    const int64_t cut = (longest + tile * ATTEND_CHUNK_MIN - 1) / (tile * ATTEND_CHUNK_MIN);
    int64_t grid = (int64_t)ATTEND_CHUNKS * ctx->n_cu + streams_units;
    grid = streams_units * cut < grid ? streams_units * cut : grid;
    grid += 8 * units;                                       // the last eight chunks' units, of which not all need be there
    rh_status ws = seq_counters(ctx);
    if (ws == RH_OK) ws = seq_scratch(ctx);
    if (ws != RH_OK) return ws;
    a.ws = (float*)ctx->seq_ws; a.count = ctx->seq_cnt;
    RH_HIP(ctx, cache->type == RH_T_F32 ? launch_attend<RH_T_F32>(ctx, a, grid, cache->dim)
                : cache->type == RH_T_BF16 ? launch_attend<RH_T_BF16>(ctx, a, grid, cache->dim) : launch_attend<RH_T_E4M3>(ctx, a, grid, cache->dim));
    return RH_OK;
}
