/*
 * rh_seq.h - operators of a transformer's decode step over many live streams (gfx950).
 *
 * What precedes rh_select_regions on live streams is a score for every macroblock of each frame as it arrives.  A
 * predictor that remembers a stream's past runs one token per stream and frame: these are the operators of such a step.
 *   rh_cache_plan      pages of a paged key-value cache for the new tokens; block table, slots; pages of ended streams back
 *   rh_cache_write     keys and values of the new tokens into their slots
 *   rh_cache_attend    attention of one new token of every stream over the stream's cached tokens
 *   rh_norm_residual   residual addition and root-mean-square norm, output also in 8 bits with a scale a row
 *   rh_matvec_packed   products of a few rows with weights in 4 bits that share a scale by 32
 * They take a context of rh.h and follow its conventions: device pointers, caller-owned buffers, all work on the context's
 * stream, arguments checked before any launch, rh_last_error.  They use neither the context's network nor its capacities,
 * and count in no class of rh_profile_read.  Sums, softmax statistics and norms are held in 32 bits.
 * Scratch memory of rh_cache_attend and rh_matvec_packed (68 MB on 256 CUs) and a few counters, of rh_cache_plan too, belong to the context: the first call that wants
 * them allocates them and waits for the stream, and no later one does.  Graphs may be recorded once an rh_cache_attend or rh_matvec_packed call of the context has been made
 * (RH_E_STATE where a captured call would have to allocate).  Since calls share this memory, those of one context must not overlap on two streams, replays of
 * a graph that recorded them among them: use a context for each, or let one wait for the other.
 */
#ifndef RH_SEQ_H
#define RH_SEQ_H

#include "rh.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { RH_T_F32 = 0, RH_T_BF16 = 1, RH_T_E4M3 = 2 };   /* element types; e4m3: 8 bits, largest 448, no infinity */

#define RH_SEQ_MAX_STREAMS 2048                        /* of one rh_cache_plan or rh_cache_attend call */
#define RH_SEQ_MAX_DIM 256                             /* head size: a multiple of 32 up to this       */
#define RH_SEQ_MAX_COLS 32768                          /* of rh_norm_residual                          */

/*
 * A paged cache: n_pages pages of `page` tokens, each with `heads` keys and values of `dim` elements.  Element d of head h
 * of token t of page p lies at k + p*k_stride[0] + t*k_stride[1] + h*k_stride[2] + d (strides in elements, so
 * both [page][token][head][dim] and [page][head][token][dim] are taken).  k and v are 16-byte aligned and their strides
 * multiples of 16 bytes; n_pages*page < 2^31 (the elements may pass 2^32).  A slot is p*page + t.
 * RH_T_E4M3: an element stands for its value times the scale of its token and head, k_scale / v_scale f32
 * [n_pages][heads][page]; NULL for the other types.
 */
typedef struct {
    void *k, *v;
    float *k_scale, *v_scale;
    int64_t k_stride[3], v_stride[3];
    int32_t type, n_pages, page, heads, dim;
} rh_kv_cache;

/*
 * Room in the cache for the next tokens of n_streams streams (at most RH_SEQ_MAX_STREAMS).  One launch.
 *   n_new (dev) i32 [n_streams]: tokens that join; negative: the stream has ended.
 *   lengths (dev) i32 [n_streams]: tokens that a stream has; block_table (dev, in/out) i32 [n_streams][max_pages]: its pages.
 *   free_pages (dev, in/out) i32 [n_pages] and free_count (dev) i32 [1]: a stack of the pages nobody has.
 * In this order: the pages of the ended streams, streams and pages ascending, are put on the stack (their length becomes
 * 0, their table entries stay).  Then the streams are served in order; one is granted its tokens when its pages fit its
 * table row, when it needs no page or the running sum of pages asked for (by it and the streams before it whose pages fit their rows)
 * is within the stack, and when the running sum of tokens asked for likewise is within n_slots.  Otherwise it gets none
 * and keeps its length: new_off tells.  Pages come from the top of the stack down.
 *   slots (dev out) i32 [n_slots]: the slot of every granted token, streams in order; -1 behind the last.
 *   new_off (dev out) i32 [n_streams + 1]: where each stream's slots begin; new_off[n_streams] = tokens granted.
 *   new_lengths (dev out) i32 [n_streams], new_count (dev out) i32 [1]: lengths and stack height afterwards; may be `lengths`
 *   and `free_count` themselves.  Of the table only the entries of granted pages are written.
 * Lengths below 0 count as 0, lengths past the table's row as the whole row when the stream ends.  n_pages and the table's entries together stay below 2^31.
 */
rh_status rh_cache_plan(rh_ctx* ctx, const int32_t* n_new, const int32_t* lengths, int32_t n_streams, int32_t page,
                        int32_t n_pages, int32_t max_pages, int32_t* block_table, int32_t* free_pages,
                        const int32_t* free_count, int32_t* slots, int32_t n_slots, int32_t* new_off,
                        int32_t* new_lengths, int32_t* new_count);

/*
 * Keys and values of n tokens into their slots.  k, v (dev): `type` (RH_T_F32 or RH_T_BF16), element (token, head, d) at
 * token*stride[0] + head*stride[1] + d.  slots (dev) i32 [n]; a slot outside [0, n_pages*page) is skipped (-1: a token that got no room).
 * Rounded to nearest even where the cache has fewer bits; RH_T_E4M3: scale = max(largest magnitude of the head, 2^-100) * (1/448),
 * element = value / scale rounded to e4m3; 1/448, product and quotient are each rounded to fp32.  RH_E_UNIMPLEMENTED: bf16 values into an fp32 cache.
 * Slots of one call must differ.
 */
rh_status rh_cache_write(rh_ctx* ctx, const rh_kv_cache* cache, const void* k, const int64_t k_stride[2], const void* v,
                         const int64_t v_stride[2], int32_t type, const int32_t* slots, int32_t n);

/*
 * Attention of one new token of every stream: out = sum_t softmax_t(scale * q.k_t) v_t over the tokens
 * t in [max(0, lengths[b] - window), lengths[b]) of stream b (window 0: all), q head h with cache head h / (q_heads / cache->heads).
 *   q (dev): `type`, element (b, h, d) at b*q_stride[0] + h*q_stride[1] + d.  out (dev) [n_streams][q_heads][dim], the same type, 16-byte aligned.
 *   lse (dev out, may be NULL): f32 [n_streams][q_heads], log sum exp(scale * q.k).
 *   block_table (dev) i32 [n_streams][max_pages]; a length past the row counts as the whole row, one below 0 as 0.
 * RH_T_F32 with an fp32 cache, RH_T_BF16 with a bf16 or an e4m3 cache (RH_E_UNIMPLEMENTED otherwise).
 * A stream without tokens gives zeros and lse = -infinity, and so does one whose table entries all lie outside
 * [0, n_pages): tokens of such pages are left out.  What the cache holds beside the tokens named does not matter.
 * Sums of one call come in the same order every time: results do not change from run to run.
 */
rh_status rh_cache_attend(rh_ctx* ctx, const rh_kv_cache* cache, const void* q, const int64_t q_stride[2], int32_t type,
                          int32_t q_heads, const int32_t* block_table, int32_t max_pages, const int32_t* lengths,
                          int32_t n_streams, float scale, int32_t window, void* out, float* lse);

/*
 * Residual addition and root-mean-square norm of n_rows rows of n_cols <= RH_SEQ_MAX_COLS elements of `type` (RH_T_F32 or RH_T_BF16):
 *   s = x + residual (residual NULL: s = x),  y = s * weight / sqrt(mean(s^2) + eps)
 * with s unrounded.  Outputs, each may be NULL but not all:
 *   sum: s in `type` (may be `residual` or `x` itself);  y in `type`;
 *   y8, y8_scale (both or none): e4m3 [n_rows][n_cols] and f32 [n_rows], scale = max(largest |y| of the row, 2^-100) * (1/448), y8 = y / scale as there.
 * x, residual and sum have a row stride each (elements, >= n_cols); y and y8 are dense.  weight (dev) f32 [n_cols].
 */
rh_status rh_norm_residual(rh_ctx* ctx, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                           const float* weight, int32_t type, int32_t n_rows, int32_t n_cols, float eps, void* sum,
                           int64_t sum_stride, void* y, uint8_t* y8, float* y8_scale);

/*
 * y[m][n] = x_scale[m] * sum_k x[m][k] * w[n][k], optionally ReLU, for a few rows m: weights are read once for 16 of them (fp32), for
 * 32 (bf16, e4m3).
 *   w (dev) u8 [n_out][16*ceil(n_in/32)], 16-byte aligned: codes of 4 bits, even k in the low half; code c stands for
 *   {0, 1/2, 1, 3/2, 2, 3, 4, 6}[c & 7], negative with bit 3.  w_scale (dev) u8 [n_out][ceil(n_in/32)]: 32 codes
 *   share the factor 2^(scale - 127) (255 is not a number).  Codes past n_in do not matter.
 *   x (dev) [n_rows] rows x_stride elements apart, RH_T_F32, RH_T_BF16 or RH_T_E4M3; x_scale (dev) f32 [n_rows]
 *   or NULL for ones.  y (dev): RH_T_F32 or RH_T_BF16, rows y_stride elements apart.
 * Long rows are cut into slices that workgroups share; sums of one call come in the same order every time.
 */
rh_status rh_matvec_packed(rh_ctx* ctx, const void* x, int32_t x_type, int64_t x_stride, const float* x_scale,
                           const uint8_t* w, const uint8_t* w_scale, int32_t n_rows, int32_t n_out, int32_t n_in,
                           int32_t relu, void* y, int32_t y_type, int64_t y_stride);

#ifdef __cplusplus
}
#endif
#endif /* RH_SEQ_H */
