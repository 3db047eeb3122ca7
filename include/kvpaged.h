/* kvpaged.h - the operators of one serving step over a paged KV cache.
 *
 * kvcfg.h decides how much memory each tier of an LLM service's KV cache gets;
 * the calls here fill and read such a cache on the GPU, in blocks of the size
 * the traces are cut into (16 or 64 tokens), so that a chosen configuration
 * can be run and the time of a recomputed token (kv_cost_model's
 * t_prefill_per_token) measured on the card instead of assumed:
 *
 *   kv_paged_plan       block tables, cache slots, positions and the
 *                       attention's work list from the requests' lengths
 *                       (once per step, for every layer)
 *   kv_rope_apply       rotary positions on a tensor of heads, or the gradient
 *   kv_paged_append     rotary positions on queries and keys, keys and values
 *                       written into the cache
 *   kv_paged_attention  attention of the step's new tokens over their
 *                       requests' blocks, single tokens and long chunks alike
 *
 * Conventions are those of kvcfg.h: KV_OK or a negative kv_status with
 * kv_last_error(), arguments checked before any device work, no C++ exception
 * crosses, device work enqueued on `stream` and outputs valid once it has
 * completed.  No call here allocates device memory, waits for the device or
 * copies to the host, except kv_rope_create and kv_rope_free; all may be
 * recorded into a HIP graph.  What only the device knows (lengths, tables,
 * slots) cannot be refused by a call: out-of-range values are skipped or
 * masked as said at each field, and reported in kv_paged_batch.result.
 *
 * Cache layout, per layer:
 *   K  [n_blocks][kv_heads][block_size][head_dim]
 *   V  [n_blocks][kv_heads][head_dim][block_size]
 * V is kept transposed: the product of the softmax weights with V sums over
 * keys, and the matrix instructions take runs of the summed index.
 */
#ifndef KVPAGED_H
#define KVPAGED_H

#include "kvcfg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  KV_DT_FP8 (e4m3: 4 exponent bits, 3 mantissa bits, no
 * infinities, largest 448) is a cache type only: the value is the stored
 * number times the scale of its key/value head. */
enum { KV_DT_BF16 = 0, KV_DT_F16 = 1, KV_DT_FP8 = 2 };

enum {
  KV_PAGED_MAX_REQ = 4096,       /* requests of a step                        */
  KV_PAGED_MAX_TOKENS = 524288   /* new tokens of a step                      */
};

/* ---- rotary positions -------------------------------------------------- */

/* Which elements form a pair: i and i + rot_dim/2, or 2i and 2i + 1. */
enum { KV_ROPE_HALF = 0, KV_ROPE_INTERLEAVED = 1 };

/* Frequencies f_i = base^(-2i/rot_dim) radians a token, and for contexts
 * longer than the trained one:
 *   LINEAR    f_i / factor
 *   BY_PARTS  g*f_i + (1-g)*f_i/factor, where g rises from 0 to 1 as the turns
 *             the pair makes over original_len tokens (original_len*f_i/2pi)
 *             rise from `slow` to `fast` */
enum { KV_ROPE_PLAIN = 0, KV_ROPE_LINEAR = 1, KV_ROPE_BY_PARTS = 2 };

typedef struct kv_rope_desc {
  uint32_t rot_dim;      /* elements of a head that turn (its first ones): a
                            multiple of 16, 16..256                           */
  uint32_t layout;       /* KV_ROPE_HALF or KV_ROPE_INTERLEAVED               */
  uint32_t scaling;      /* KV_ROPE_PLAIN, _LINEAR or _BY_PARTS               */
  uint32_t original_len; /* BY_PARTS: trained context, > 0                    */
  double base;           /* > 1                                               */
  double factor;         /* LINEAR, BY_PARTS: >= 1                            */
  double fast, slow;     /* BY_PARTS: fast > slow >= 0                        */
  double magnitude;      /* multiplies the turned elements, in 32 bits: finite
                            and nonzero there                                 */
} kv_rope_desc;

typedef struct kv_rope kv_rope; /* opaque: the pairs' frequencies, on the current device */

/* Makes a rotation, usable on every stream of the current device; allocates
 * and waits.  KV_ERR_INVALID for a value outside the ranges above. */
kv_status kv_rope_create(const kv_rope_desc* desc, kv_rope** out);

/* Frees a rotation once the device has finished with it (waits); NULL is
 * accepted, a pointer that is no live rotation is KV_ERR_INVALID. */
kv_status kv_rope_free(kv_rope* r);

/* A tensor [tokens][heads][head_dim]: elements of a head are contiguous,
 * tokens and heads at any stride (in elements, multiples of 8); ptr 16-byte
 * aligned. */
typedef struct kv_heads_view {
  void* ptr;
  int64_t token_stride, head_stride;
} kv_heads_view;

/* y = rotation of x at positions pos, per pair (a, b) with angle p*f_i and
 * magnitude m: (m*(a*cos - b*sin), m*(a*sin + b*cos)); backward: the same with
 * the angle negated, the gradient of x for a gradient of y.  Elements past
 * rot_dim are copied.  Frequencies have the 53 bits of a double and angles are
 * reduced modulo a turn without further error: they are off by less than 2^-22
 * turns at any position.  The products are in 32 bits, rounded once.
 *   dtype     KV_DT_BF16 or KV_DT_F16
 *   x, y      views; y may be x itself (same pointer and strides), otherwise
 *             they must not overlap
 *   pos       device int32 [n_tokens], any value
 *   head_dim  a multiple of 16, rot_dim..256
 * n_tokens == 0 or n_heads == 0 is a no-op. */
kv_status kv_rope_apply(const kv_rope* r, uint32_t dtype, kv_heads_view x, kv_heads_view y,
                        const int32_t* pos, uint32_t n_tokens, uint32_t n_heads,
                        uint32_t head_dim, int backward, void* stream);

/* ---- one step's batch ---------------------------------------------------- */

/* One step: request r has ctx_len[r] tokens in the cache already (a reused
 * prefix, earlier steps) and brings new_len[r] tokens; the step's tokens are
 * the requests' new tokens one after another.  All pointers are device memory;
 * the arrays after `table` are written by kv_paged_plan and read by the other
 * calls of the step. */
typedef struct kv_paged_batch {
  uint32_t n_req;       /* 1..KV_PAGED_MAX_REQ                                */
  uint32_t max_tokens;  /* 1..KV_PAGED_MAX_TOKENS: length of slot and pos; may
                           exceed the step's tokens                           */
  uint32_t max_new;     /* no request brings more; 0 = max_tokens.  Steps of
                           single tokens should say 1                         */
  uint32_t block_size;  /* 16, 32, 64, 128 or 256 tokens                      */
  uint32_t max_blocks;  /* columns of table; max_blocks*block_size <= 2^30    */
  uint32_t q_heads;     /* a multiple of kv_heads; query head h reads
                           key/value head h / (q_heads/kv_heads)              */
  uint32_t kv_heads;    /* 1..1024                                            */
  uint32_t head_dim;    /* 64, 128 or 256                                     */
  uint32_t window;      /* a token sees itself and the window-1 before it; 0 =
                           every earlier token                                */
  uint32_t n_free;      /* entries of free_list                               */
  const int32_t* ctx_len;   /* [n_req]                                        */
  const int32_t* new_len;   /* [n_req]                                        */
  int32_t* table;           /* [n_req][max_blocks] block of each run of
                               block_size tokens; a negative entry (or one >=
                               the cache's n_blocks) is a block that is not
                               there: its keys are masked                     */
  const int32_t* free_list; /* [n_free] blocks to take, first entry first, or
                               NULL: table names the new tokens' blocks already
                               (an empty list: n_free 0 and any other address) */
  int32_t* q_start;     /* [n_req+1] first token of each request, then the
                           step's number of tokens                            */
  int32_t* kv_len;      /* [n_req] ctx_len + new_len                          */
  int64_t* slot;        /* [max_tokens] cache slot (block*block_size + offset)
                           of each token; -1: no block, or past the last token */
  int32_t* pos;         /* [max_tokens] position in its request; 0 past the last */
  int32_t* result;      /* [4] tokens of the step, blocks needed, blocks taken,
                           KV_PLAN_* flags                                    */
  void* work;           /* work list and partial results, 256-byte aligned; one
                           step's calls at a time                             */
  uint64_t work_bytes;  /* at least kv_paged_work_bytes                       */
} kv_paged_batch;

/* result[3]: what was wrong with the device's data. */
enum {
  KV_PLAN_BAD_LENGTH = 1, /* a length is negative, exceeds max_new, or the sum
                             exceeds max_blocks*block_size: taken as 0, 0      */
  KV_PLAN_TOKENS = 2,     /* the new tokens exceed max_tokens: the request that
                             goes past it and all later ones bring none        */
  KV_PLAN_BLOCKS = 4      /* free_list is too short: the last requests' tokens
                             without a block get slot -1 and table entry -1    */
};

/* Bytes of batch->work for these sizes (pointers are not looked at). */
kv_status kv_paged_work_bytes(const kv_paged_batch* b, uint64_t* bytes);

/* Fills the batch's arrays.  A request takes new blocks for the runs of tokens
 * that begin at or after ctx_len; the block a context ends inside is written
 * on (the caller makes it the request's own first).  Whole numbers; a repeated
 * call on the same inputs gives the same outputs.  KV_ERR_INVALID for a NULL
 * pointer (free_list aside), a misaligned one, or sizes outside the ranges. */
kv_status kv_paged_plan(const kv_paged_batch* b, void* stream);

/* ---- the cache ----------------------------------------------------------- */

typedef struct kv_paged_cache {
  void* k;               /* device, 16-byte aligned                           */
  void* v;
  int64_t k_block_stride; /* elements from one block to the next, a multiple of
                             16 and at least kv_heads*block_size*head_dim      */
  int64_t v_block_stride;
  uint32_t n_blocks;     /* >= 1                                              */
  uint32_t dtype;        /* KV_DT_*                                           */
  const float* k_scale;  /* device [kv_heads], > 0: KV_DT_FP8 only; NULL = 1  */
  const float* v_scale;
} kv_paged_cache;

/* Writes the step's keys and values into their slots, and turns queries and
 * keys by their positions on the way.
 *   q, q_out  views of q_heads heads, or q.ptr NULL: no queries; q_out may be q
 *   k, v      views of kv_heads heads
 *   rope      or NULL: nothing turns (queries are then copied)
 *   dtype     of q, k and v: KV_DT_BF16 or KV_DT_F16; a 16-bit cache must have
 *             the same type
 * Into a KV_DT_FP8 cache goes value/scale rounded to nearest even, values past
 * +-448 as +-448, NaN as NaN.  Tokens without a slot, or with one outside the
 * cache, are not written; rows past the step's last token are left alone.  No
 * two tokens may have one slot. */
kv_status kv_paged_append(const kv_paged_batch* b, const kv_paged_cache* c, const kv_rope* rope,
                          uint32_t dtype, kv_heads_view q, kv_heads_view q_out, kv_heads_view k,
                          kv_heads_view v, void* stream);

/* out[t][h] = sum_j softmax_j(scale * q[t][h].K[j]) V[j] over the keys j that
 * token t sees: its request's positions up to its own, within the window, in
 * blocks that are there.  lse[t][h] = log sum_j exp(scale * q.K[j]).  A token
 * that sees nothing gets zeros and -inf.  Masked keys and values count for
 * nothing whatever they hold.  Of what is seen, a score of -inf weighs nothing
 * (no other: as if nothing was seen), one of +inf or NaN leaves NaN in out and
 * lse.  Products are on the matrix cores with 32-bit sums; softmax statistics
 * are in 32 bits; the weights are rounded to the queries' type for the second
 * product.  Sums are taken with weights of up to 2^14 before the division, so
 * values past some 10^30 may leave the 32-bit range.  Results do not depend on
 * timing.
 *   q, out    views of q_heads heads; out must not overlap q (the
 *             same pointer is KV_ERR_INVALID)
 *   lse       device float [max_tokens][q_heads] or NULL
 *   scale     > 0 and finite
 * Rows past the step's last token are left alone.  The batch must have been
 * planned on this stream (or waited for) with the same sizes, window included:
 * with a work list for other sizes the call writes nothing. */
kv_status kv_paged_attention(const kv_paged_batch* b, const kv_paged_cache* c, uint32_t dtype,
                             kv_heads_view q, kv_heads_view out, float* lse, float scale,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KVPAGED_H */
