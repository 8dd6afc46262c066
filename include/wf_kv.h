/*
 * wf_kv.h -- C ABI of the paged 4-bit key/value cache of one replica.
 *
 * The scheduler (wf_plan.h) decides which activations a replica serves next;
 * serving them means giving their requests cache blocks, storing the keys and
 * values of their new tokens, and attending to what is stored (Sec. 4:
 * replicas serve with continuous batching; Eq. 11 counts what the cache
 * holds as the activation's memory).  These calls do that on the GPU, for one
 * step of a batch of requests:
 *
 *   wf_kv_step    blocks and slots of the step's tokens, from the requests'
 *                 lengths;
 *   wf_kv_store   per layer: norm and rotation of queries and keys, queries
 *                 out, keys and values into the cache;
 *   wf_kv_attend  per layer: attention of the step's queries over the cache;
 *   wf_kv_load    cached tokens back as values.
 *
 * Rows and tokens.  A batch has n_rows rows, one per request; row r brings
 * new_tokens[r] tokens.  The tokens of all rows are packed in row order, row
 * r's at q_off[r] .. q_off[r+1]-1.  A token has a position in its request and
 * a slot in the cache: block * block_tokens + offset in the block; a slot
 * below 0 stores nothing.
 *
 * Cache.  n_blocks blocks of block_tokens tokens, one buffer per layer.  Block
 * b and kv head h have one cell of B * (D + 4) bytes (B = block_tokens, D =
 * head_dim) at ((b * kv_heads) + h) * B * (D + 4):
 *   key codes    [B][D/2]  byte j: channel 2j in the low nibble, 2j+1 high
 *   value codes  [D/2][B]  byte (r, t) of token t: channel r low, r + D/2 high
 *   key scales   [B] bf16
 *   value scales [B] bf16
 * A code is E2M1: bit 3 the sign, bits 2..0 one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.
 * A stored value is its code's value times the scale of its token and head.
 * The scale is bf16(fp32(largest magnitude * fp32(1/6))), rounded to nearest even;
 * a code is the nearest one to value / scale, ties to the even code, above 6
 * taken as 6.  A vector with an infinity or a NaN gets a NaN scale: it stands
 * for NaN in every channel.
 *
 * Conventions are those of wf_plan.h: C functions that never throw and return
 * a wf_status; caller-owned DEVICE buffers of the context's GPU, contiguous
 * unless a stride is an argument, alive until the work queued on hip_stream
 * (NULL = the default stream) is done; argument errors are found before
 * anything is queued and change nothing.  No call allocates, copies to the
 * host or synchronises, except create and destroy, so all others may be
 * captured in a HIP graph.  What lies in device arrays cannot be checked by
 * the host: block ids, slots, positions, lengths or offsets outside their
 * range give unspecified results without touching memory outside the arrays.
 * A context is not thread-safe.  Calls of one context on different streams may
 * run at the same time (on data of their own): each of the first
 * WF_KV_ATTEND_STREAMS streams that wf_kv_attend is called on has a work area of
 * the context for good (allocated at create); on further streams long rows of few
 * queries take longer, as their tokens are not shared out.  A captured call keeps the area of
 * the stream that it was captured on: replays of such graphs must not run at the same
 * time as each other or as calls on that stream.
 */
#ifndef WF_KV_H
#define WF_KV_H

#include "wf_plan.h"

#ifdef __cplusplus
extern "C" {
#endif

#define WF_KV_MAX_ROWS 65536        /* rows of a batch                         */
#define WF_KV_MAX_TOKENS (1 << 24)  /* packed tokens of a step                 */
#define WF_KV_MAX_HEADS 1024        /* query heads                             */
#define WF_KV_MAX_BLOCKS (1 << 30)  /* blocks of a cache                       */
#define WF_KV_ATTEND_STREAMS 8      /* streams with a work area of their own   */
#define WF_KV_MAX_WIDTH (1 << 22)   /* blocks of a row, of at most 2^30 tokens     */

enum { WF_KV_BF16 = 0, WF_KV_F16 = 1 };

/* Geometry of a cache and the heads that use it. */
typedef struct {
  int32_t q_heads;       /* a multiple of kv_heads, 1..WF_KV_MAX_HEADS          */
  int32_t kv_heads;      /* >= 1; query head i uses kv head i / (q_heads / kv_heads) */
  int32_t head_dim;      /* D: 64, 128 or 256                                   */
  int32_t block_tokens;  /* B: 16, 32, 64, 128 or 256                           */
  int32_t n_blocks;      /* 1..WF_KV_MAX_BLOCKS                                 */
  int32_t max_blocks;    /* width of the block table: most blocks of a row      */
  int32_t dtype;         /* WF_KV_BF16 or WF_KV_F16: queries, keys, values and
                            norm weights in, queries, values and outputs out    */
} wf_kv_desc;

typedef struct wf_kv_ctx wf_kv_ctx; /* opaque; geometry and work area */

/* Bytes of one layer's cache.  Host only.  The message of an error is in
 * wf_kv_last_error(NULL). */
wf_status wf_kv_cache_bytes(const wf_kv_desc *desc, int64_t *bytes);

/* Create a context on HIP device `hip_device`; it copies *desc and allocates
 * the work areas of wf_kv_attend (272 MiB).  On failure *out is NULL and
 * wf_kv_last_error(NULL) describes the error. */
wf_status wf_kv_ctx_create(int hip_device, const wf_kv_desc *desc, wf_kv_ctx **out);

/* Free the context (NULL is a no-op).  Work queued on it must have completed. */
void wf_kv_ctx_destroy(wf_kv_ctx *ctx);

/* As wf_plan_last_error, for this part of the library. */
const char *wf_kv_last_error(const wf_kv_ctx *ctx);

/*
 * Block tables and slots of one step.  Row r holds len_in[r] tokens in the
 * blocks table[r][0 .. ceil(len_in[r] / B)).  new_tokens[r] >= 0 asks for that many
 * more; new_tokens[r] < 0 releases the row.  Free blocks are in a ring of n_blocks
 * ids: pool_in[0] is the index of the first, pool_in[1] their number.
 *   - A row needs ceil((len + new) / B) - ceil(len / B) blocks.  Rows are
 *     granted in row order: a row is granted when it needs none, or when its need
 *     and that of all rows before it (granted or not) fit in the free blocks.
 *     A row that would be longer than max_blocks blocks is refused and
 *     its need not counted.  granted[r] is 1 or 0 (0 also for a released row).
 *   - Granted rows take blocks from the front of the ring in row order, into the
 *     next entries of table[r].
 *   - Blocks of released rows go to the end of the ring in row order; they can
 *     be taken from the next step on.  The row's table entries stay as they are.
 *   - len_out[r] = len + new (granted), 0 (released), len (refused); pool_out
 *     likewise.  The old arrays are left as they were: a caller keeps two of
 *     each and swaps them.
 *   - q_off[0 .. n_rows] are the offsets of the rows' packed tokens (refused rows
 *     included); token i of row r gets pos = len_in[r] + i and its slot, -1
 *     when the row is refused.  Entries from q_off[n_rows] to n_tokens get pos
 *     0 and slot -1; tokens past n_tokens are left out.
 * Arrays: new_tokens, len_in, len_out int32 [n_rows]; pool_in, pool_out int32
 * [2]; ring int32 [n_blocks]; table int32 [n_rows][max_blocks]; q_off int32
 * [n_rows + 1]; slot int64 [n_tokens]; pos int32 [n_tokens]; granted uint8
 * [n_rows].  len_out and pool_out must not be len_in and pool_in.
 */
wf_status wf_kv_step(wf_kv_ctx *ctx, const int32_t *new_tokens, int32_t n_rows, int32_t n_tokens,
                     const int32_t *len_in, int32_t *len_out, const int32_t *pool_in,
                     int32_t *pool_out, int32_t *ring, int32_t *table, int32_t *q_off,
                     int64_t *slot, int32_t *pos, uint8_t *granted, void *hip_stream);

/* How wf_kv_store norms and rotates. */
typedef struct {
  const void *q_weight;    /* [D] norm weight of the queries, NULL: no norm     */
  const void *k_weight;    /* [D] norm weight of the keys, NULL: no norm        */
  float eps;               /* finite, >= 0                                      */
  int32_t rot_dim;         /* rotated channels: a multiple of 16, 0..D          */
  int32_t interleaved;     /* 0: pairs (c, c + rot_dim/2), 1: pairs (2c, 2c+1)  */
  int32_t n_pos;           /* rows of cos_sin                                   */
  const float *cos_sin;    /* [n_pos][rot_dim]: rot_dim/2 cosines, then sines;
                              may be NULL when rot_dim is 0                     */
} wf_kv_norm_rope;

/*
 * Queries and keys x of each head are normed, x * rsqrt(mean(x^2) + eps) * w,
 * and rotated by their token's position: (a, b) -> (a cos - b sin, b cos + a
 * sin).  Queries are written to q_out [n_tokens][q_heads][D], rounded once; keys
 * and values go into the cache at their slots.  q [n_tokens][q_heads][D], k and
 * v [n_tokens][kv_heads][D]: heads contiguous, tokens q_stride, k_stride and
 * v_stride elements apart (multiples of 8, and the addresses of 16 bytes), so
 * that slices of one projection can be passed.  pos int32 [n_tokens] (may be
 * NULL when rot_dim is 0), slot int64 [n_tokens].  Two tokens must not have
 * the same slot.  All arithmetic is in fp32.
 */
wf_status wf_kv_store(wf_kv_ctx *ctx, const void *q, const void *k, const void *v,
                      int64_t q_stride, int64_t k_stride, int64_t v_stride, int32_t n_tokens,
                      const wf_kv_norm_rope *how, const int32_t *pos, const int64_t *slot,
                      void *q_out, uint8_t *cache, void *hip_stream);

/* The values that the cache holds at slot[0 .. n_tokens): k_out and v_out
 * [n_tokens][kv_heads][D], code value times scale rounded to the context's
 * type, at most its largest finite value; zeros for a slot outside the cache. */
wf_status wf_kv_load(wf_kv_ctx *ctx, const uint8_t *cache, const int64_t *slot, int32_t n_tokens,
                     void *k_out, void *v_out, void *hip_stream);

/*
 * out[t][i] = sum_j p_j v_j, p = softmax_j(scale * q[t][i] . k_j), over the
 * cached tokens j of t's row with j < kv_len[row], j <= pos[t] and, when window
 * > 0, j > pos[t] - window.  A query that sees no token gets 0.  q
 * [n_tokens][q_heads][D], tokens q_stride elements apart (a multiple of 8; the
 * address of 16 bytes); out [n_tokens][q_heads][D]; table int32 [n_rows][max_blocks];
 * kv_len int32 [n_rows]; q_off int32 [n_rows + 1]; pos int32 [n_tokens].  Tokens
 * from q_off[n_rows] on are not written.
 * max_q and max_kv are hints for the launch: the most queries and the most cached
 * tokens of a row (0: not known).  Results are right whatever they are, to the
 * roundings of the kernel taken; unknown, too low or too high ones cost time.
 * The kernel is chosen for the whole call, by its longest row: single tokens beside a
 * long prompt take less time in a call of their own.
 * Products are of 16-bit values with fp32 sums; the softmax is fp32, its
 * probabilities times the value scales are rounded to the 16-bit type.  Sums are
 * divided by the softmax's total at their end: with bf16, values must stay below
 * about 1e36 / (tokens seen) for them to be finite.  With f16 the largest
 * probability times scale is moved to the upper part of the type's range first,
 * so that small values keep as many bits as large ones.
 */
wf_status wf_kv_attend(wf_kv_ctx *ctx, const void *q, int64_t q_stride, int32_t n_tokens,
                       const uint8_t *cache, const int32_t *table, const int32_t *kv_len,
                       const int32_t *q_off, const int32_t *pos, int32_t n_rows, float scale,
                       int32_t window, int32_t max_q, int32_t max_kv, void *out, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* WF_KV_H */
