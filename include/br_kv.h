/*
 * What a worker does with the requests that br.h has bound to it, for MI355X (gfx950): C ABI.
 *
 * The router's unit of load is a worker's cached tokens (L_g, br.h): what the attention of one decode step reads.  This
 * part holds those tokens.  Per decode step and worker:
 *   br_kv_step    block tables and slot maps from the lengths that stay and the tokens that come
 *   br_kv_append  keys and values of the new tokens into the cache: 8 bits, a scale for each block of tokens and head
 *   br_kv_attend  attention of the new tokens over their requests' cached tokens
 *   br_kv_read    keys and values of cached tokens back out (hand-over of a request to another worker)
 * A context serves n_workers workers side by side (several DP ranks of a replay on one GPU, or one).  The tables are one
 * per worker for all layers of a model; the cache of each layer is memory of the caller's (br_kv_layer).
 *
 * Conventions are br.h's: every pointer inside the argument structs is a DEVICE pointer, the structs are host memory; the
 * library allocates and frees no device memory and never synchronises; all work is enqueued on the context's stream and
 * buffers stay alive until it ran; BR_OK or a negative code of br.h comes back, nothing is printed, nothing aborts.  No
 * call but br_kv_init allocates host memory; all of them may be captured into a graph.  Calls on one context
 * share its workspace: from several threads they are serialised by the caller.
 * The context's GPU has to be the current device of the calling thread, as for br.h's calls.  Memory that other streams have written or
 * will read is ordered against the context's stream by the caller (events); the library adds no waits.
 *
 * What a call reads on the device stays as it is until the call has run.  An attention whose lengths or counts are changed under it leaves outputs
 * that are not said, and so may those behind it up to the next br_kv_step.
 *
 * What is read on the device is checked there and never leads outside a buffer: lengths, block ids, slots, starts and
 * counts out of range are clamped or skipped as each call says.
 *
 * Layout of a layer's cache, `block` = ((w * n_blocks + id) * n_kv_heads + h) for block id of worker w and head h:
 *   k       [block][block_tokens][head_dim]  bytes    k_scale [block] float
 *   v       [block][head_dim][block_tokens]  bytes    v_scale [block] float
 * (values run along the tokens: the attention's second product takes 16 tokens of a channel per load).
 * A byte is a code: BR_KV_INT8 two's complement, BR_KV_E4M3 the 8-bit float of 4 exponent and 3 mantissa bits without
 * infinities (codes of NaN are not written and may not be read; a NaN is carried by the scale).  Value = code * scale.
 */
#ifndef BR_KV_H
#define BR_KV_H

#include <stdint.h>

#include "br.h"

#ifdef __cplusplus
extern "C" {
#endif

#define BR_KV_MAX_WORKERS 16777215
#define BR_KV_MAX_ROWS 1024
#define BR_KV_MAX_BLOCKS 262144      /* blocks of a worker */
#define BR_KV_MAX_LEN 1048576        /* tokens that a row's table may span */
#define BR_KV_MAX_HEADS 1024         /* query heads */
#define BR_KV_MAX_STRIDE 8388608     /* elements between a token's keys (values) and the next one's */
#define BR_KV_NSTATS 8

enum { BR_KV_INT8 = 0, BR_KV_E4M3 = 1 };             /* fmt: codes of the cache */
enum { BR_KV_F16 = 0, BR_KV_BF16 = 1, BR_KV_F32 = 2 }; /* dtype: keys, values, queries, outputs (attention: F16 or BF16) */

/* status of a row after br_kv_step */
enum {
  BR_KV_TAKEN = 0,     /* what was asked for */
  BR_KV_NO_BLOCKS = 1, /* the worker has too few free blocks for this row and those before it */
  BR_KV_TOO_LONG = 2,  /* the row would need more than max_blocks blocks */
  BR_KV_NO_ROOM = 3    /* the token list is too short for this row and those before it */
};

/* slots of a worker's stats block (int64 each), after the step */
enum {
  BR_KV_ST_TOKENS = 0, /* cached tokens: the worker's load L_g */
  BR_KV_ST_USED = 1,   /* blocks in use */
  BR_KV_ST_FREE = 2,   /* blocks free */
  BR_KV_ST_ROWS = 3,   /* rows that hold tokens */
  BR_KV_ST_ADDED = 4,  /* tokens in the token list */
  BR_KV_ST_REFUSED = 5,   /* rows whose tokens were refused, for any reason */
  BR_KV_ST_NO_BLOCKS = 6, /* ... for want of blocks */
  BR_KV_ST_TAKEN = 7      /* blocks taken in this step */
};

typedef struct br_kv_ctx br_kv_ctx; /* opaque; host object owned by the library */

typedef struct {
  int32_t n_workers;    /* 1..2^24 - 1; n_workers * rows < 2^26 */
  int32_t rows;         /* requests a worker may hold (its slot limit), 1..1024 */
  int32_t block_tokens; /* 16, 32, 64 or 128 */
  int32_t n_blocks;     /* blocks of each worker, 1..262144 */
  int32_t max_blocks;   /* entries of a row's table; max_blocks * block_tokens <= 2^20 */
  int32_t n_kv_heads;   /* >= 1 */
  int32_t n_q_heads;    /* a multiple of n_kv_heads, at most 1024: heads h*g .. h*g+g-1 read key head h */
  int32_t head_dim;     /* 64, 96, 128, 192 or 256 */
  int32_t fmt;          /* BR_KV_INT8 or BR_KV_E4M3 */
  int32_t pad;
  void *stream;         /* hipStream_t, borrowed for the life of the context (NULL = default) */
  void *workspace;      /* device memory, >= br_kv_workspace_bytes() bytes, 256-byte aligned, borrowed */
  uint64_t workspace_bytes;
} br_kv_config;

/*
 * Optional requests held at the start: lens [n_workers][rows], table [n_workers][rows][max_blocks]; entry j of a row
 * holds its tokens j*block_tokens and on.  A block belongs to one row.  Lengths are clamped to what a table spans; ids
 * outside [0, n_blocks) count as no block (-1).  Copied by br_kv_init.
 */
typedef struct {
  const int32_t *lens;
  const int32_t *table;
} br_kv_state;

/*
 * One step's requests.  Both [n_workers][rows].  keep: tokens that stay in the row (clamped to what it holds; < 0: all of
 * them): its length for a request that goes on, less where drafted tokens were rejected, 0 where the request is gone.
 * add: tokens that come (values < 0 count as 0).  keep 0 with add > 0 starts a new request in the row.
 */
typedef struct {
  const int32_t *keep;
  const int32_t *add;
} br_kv_lengths;

/*
 * Outputs of a step; every pointer may be NULL to skip that output.
 *  slot  [n_workers][token_cap]  where each new token goes in its worker's cache (block id * block_tokens + offset),
 *                                rows in order, a row's tokens in order; -1 behind the last
 *  pos   [n_workers][token_cap]  its position in its request; -1 behind the last
 *  start [n_workers][rows]       where the row's tokens begin in the flat list (worker w's begin at w * token_cap)
 *  count [n_workers][rows]       tokens that the row has got: add, or 0 if refused
 *  status [n_workers][rows]      BR_KV_TAKEN, ...
 *  stats [n_workers][BR_KV_NSTATS]
 */
typedef struct {
  int32_t *slot;
  int32_t *pos;
  int32_t *start;
  int32_t *count;
  int32_t *status;
  int64_t *stats;
  int32_t token_cap; /* >= 0: room in a worker's token list; a step never adds more */
  int32_t pad;
} br_kv_step_out;

/* One layer's cache; 16-byte aligned. */
typedef struct {
  uint8_t *k;
  uint8_t *v;
  float *k_scale;
  float *v_scale;
} br_kv_layer;

/*
 * Tokens in and out of the cache.  Element (t, h, d) of k is k[t * k_token + h * k_head + d]; the same for v.
 * slot [n_workers][n_tokens], n_tokens per worker; t runs over n_workers * n_tokens.  Slots outside the worker's cache
 * (-1) are skipped by br_kv_append and read as zeros by br_kv_read.
 */
typedef struct {
  void *k;
  void *v;
  const int32_t *slot;
  int64_t k_token, k_head, v_token, v_head; /* k_token and v_token in 0 .. BR_KV_MAX_STRIDE - 1 (of one token: anything) */
  int32_t n_tokens; /* >= 0; n_workers * n_tokens at most 2^31 - 257 */
  int32_t dtype;    /* BR_KV_F16, BR_KV_BF16 or BR_KV_F32 */
} br_kv_tokens;

/*
 * Attention.  Element (t, h, d) of q is q[t * q_token + h * q_head + d], of out likewise; lse [n_tokens][n_q_heads] (natural
 * logarithm of the sum of e^score, may be NULL).  Row r (of n_workers * rows) has count[r] query tokens from token
 * start[r] on: the last count[r] positions of its lens[r] cached tokens.  start and count both NULL: a token for each row,
 * token r for row r.  A query at position p sees the positions j <= p, and if window > 0 those with j > p - window.
 * One that sees nothing (its row holds fewer tokens than it has queries) gets zeros and lse -infinity.  Tokens outside
 * [0, n_tokens) are skipped; those that no row names are not written.
 */
typedef struct {
  const void *q;
  void *out;
  float *lse;
  const int32_t *start;
  const int32_t *count;
  const int32_t *lens;  /* [n_workers][rows], NULL: the context's own */
  const int32_t *table; /* [n_workers][rows][max_blocks], NULL: the context's own */
  int64_t q_token, q_head, out_token, out_head;
  int32_t n_tokens;
  int32_t max_count; /* the largest count, >= 1: the tile of queries goes by it (larger counts are served, more slowly) */
  int32_t window;    /* >= 0; 0: off */
  int32_t dtype;     /* BR_KV_F16 or BR_KV_BF16: of q and out */
  float scale;       /* of the scores; finite */
  int32_t pad;
} br_kv_attention;

/* Where the tables live inside the workspace (byte offsets, int32): lens [n_workers][rows], table [n_workers][rows][max_blocks]. */
typedef struct {
  uint64_t lens, table, total_bytes;
} br_kv_layout;

/* Bytes of workspace a configuration needs (0 if the configuration is invalid). Host only. */
uint64_t br_kv_workspace_bytes(const br_kv_config *cfg);

/* Create a context: validates cfg, enqueues the kernels that clear its tables and load `init` if given. */
int32_t br_kv_init(const br_kv_config *cfg, const br_kv_state *init, br_kv_ctx **out);

/*
 * One step of every worker's tables.  With kp = keep clamped, b = block_tokens, in this order:
 *  1. blocks behind ceil(kp / b) are given back, for every row before any block is taken;
 *  2. rows with add > 0 are refused (they keep kp tokens) if ceil((kp + add) / b) > max_blocks; of the others, from the
 *     first on at which the sum of add in row order passes token_cap; of the others that need blocks, from the first on at which the sum
 *     of the blocks needed passes the number free (a row that needs none is never refused for want of them);
 *  3. blocks are taken in row order, positions ascending: the k-th taken is the k-th lowest of the free ids.
 * The tables' entries behind a row's last block are -1.  Equal inputs give equal tables.
 */
int32_t br_kv_step(br_kv_ctx *ctx, const br_kv_lengths *in, const br_kv_step_out *out);

/*
 * Writes tokens into the cache.  For each block and head that gets tokens, with a the largest magnitude among them (k and
 * v apart), top = 127 (BR_KV_INT8) or 448 (BR_KV_E4M3): the scale becomes the least power of two s >= 2^-100 with
 * a <= top * s, or that of the block's earlier tokens (the first new token is not at its offset 0) if that is larger (rounded up to a
 * power of two, if the cache was written elsewhere).  Codes are value / s rounded to nearest, ties to even; codes of the earlier tokens
 * are rescaled to the new s the same way.  A value that is not finite makes the scale NaN (the new tokens' codes 0) until the block is
 * begun again at offset 0: every value read there is NaN.  An earlier scale that is none (below 0, not finite, above 2^126) does the same.
 * Tokens of one block stand together in the list, offsets ascending by one, as br_kv_step lists them.  What a block holds
 * that occurs in two places of one call's list is not said; other blocks hold what they would without it.
 */
int32_t br_kv_append(br_kv_ctx *ctx, const br_kv_layer *layer, const br_kv_tokens *in);

/*
 * Reads tokens out of the cache: code * scale, rounded to dtype.  Slots in any order.  A block's scale that is none (below
 * zero or not finite) reads as NaN.
 */
int32_t br_kv_read(br_kv_ctx *ctx, const br_kv_layer *layer, const br_kv_tokens *out);

/*
 * out = softmax(scale * q k^T) v over the visible cached tokens.  Equal inputs give equal outputs, bit for bit.  Tokens that a
 * query does not see have no part in its result, whatever their codes and scales; the scale of a block that it does see
 * makes its result NaN if it is none (below zero or not finite), and so do queries that are not finite.
 * Arithmetic: scores and sums in 32 bits; the queries' channels, each row scaled by a power of two to a largest of 1..2, and the weights
 * e^(s - m) v_scale go to the matrix units in f16 (the codes are exact there), each off by 2^-11 of itself at most and by 2^-33 of the largest that
 * its query sees.  Tokens of which e^(s - m) is below 2^-126, m the query's largest score, may count as none.
 */
int32_t br_kv_attend(br_kv_ctx *ctx, const br_kv_layer *layer, const br_kv_attention *args);

/* Destroy the context (host memory only). NULL is allowed. */
void br_kv_free(br_kv_ctx *ctx);

/* The hipError_t of the last failed HIP call on this context (0 if none). */
int32_t br_kv_last_hip_error(const br_kv_ctx *ctx);

int32_t br_kv_get_layout(const br_kv_ctx *ctx, br_kv_layout *out);

#ifdef __cplusplus
}
#endif
#endif /* BR_KV_H */
