/*
 * ftcache.h -- C ABI of the paged key / value cache in 4 bits for AMD MI355X (gfx950), part of the same shared library as
 * ftattn.h: what a decoder keeps of its prompts, and the attention of single tokens over it.
 *
 * The cache is ONE device array of `pages` pages, owned by the caller (ftcache_page_bytes() each).  A page holds page_size
 * tokens of one sequence; a page table per sequence says which pages, in order.  In a page every key / value head has
 *
 *     key codes    [token][head_dim / 2 bytes]                   byte i: elements 2i (low 4 bits) and 2i + 1
 *     value codes  [token / 8][head_dim / 4][token % 8] 16 bits  word: elements 4j .. 4j + 3, lowest bits first
 *     parameters   [token / 8][4][token % 8] in_dtype            key scale, key minimum, value scale, value minimum
 *
 * and code c of a token and head stands for scale * c + minimum.  With lo and hi the smallest and largest of the head's
 * elements, minimum = lo, scale = (hi/15 - lo/15) rounded to in_dtype, c = ((x/2 - lo/2) / (scale/2)) rounded to the nearest
 * (ties to even) and held to 0..15, c = 0 where the scale is 0; all of it in 32 bits, so that the same input gives the same codes
 * everywhere.  A head with an element that is not finite has NaN for its scale and minimum.
 *
 * These operators carry no checksums: there is no protected form of them.
 *
 * Conventions
 *   - Every function returns FTCACHE_OK (0) or a negative error code and never throws or prints; ftcache_last_error() returns
 *     the message of the last failure.
 *   - Pointers to tokens, pool, tables and lengths are DEVICE pointers owned by the caller; the structures that carry
 *     them are HOST memory.  The calls leave the current device as it was.
 *   - ftcache_append, _read and _attend allocate nothing and are one kernel launch each on `hip_stream`: they may be recorded into a HIP
 *     graph by stream capture.  What the host cannot see is checked by the kernels: a page number outside the pool or a
 *     position outside the rotation table reads and writes nothing out of bounds and is counted (ftcache_report).  append puts nothing into the cache for
 *     such a token, and NaN into q_out and k_out where its position has no rotation; read and attend give NaN in its place.
 *   - append and read calls on one context may overlap in time; attend calls (which share the context's workspace)
 *     may not, captured graphs of them included.
 */
#ifndef FTCACHE_H
#define FTCACHE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ftcache_ctx ftcache_ctx; /* opaque, library-owned */

enum { FTCACHE_F16 = 0, FTCACHE_BF16 = 1, FTCACHE_F32 = 2 };
enum { FTCACHE_OK = 0, FTCACHE_EINVAL = -1, FTCACHE_EUNSUPPORTED = -2, FTCACHE_EHIP = -3, FTCACHE_ENOMEM = -4 };

typedef struct {
  uint32_t struct_size;     /* sizeof(ftcache_config), checked */
  int32_t heads, kv_heads;  /* heads: a multiple of kv_heads; query head h belongs to key / value head h / (heads / kv_heads) */
  int32_t head_dim;         /* 64 or 128 */
  int32_t pages;            /* of the pool, >= 1 */
  int32_t page_size;        /* tokens: a power of two, 16 to 1024 */
  int32_t in_dtype;         /* FTCACHE_F16 | FTCACHE_BF16: tokens and the cache's parameters */
  int32_t out_dtype;        /* result of attend: FTCACHE_F32, or in_dtype */
  int32_t rotary_dim;       /* elements of a head that are rotated: a multiple of 16 up to head_dim; 0 selects head_dim */
  int32_t interleaved;      /* 0: element a is rotated with a + rotary_dim/2; 1: element 2a with 2a + 1 */
  float softmax_scale;      /* <= 0 selects 1/sqrt(head_dim) */
  int32_t max_batch;        /* sequences of an attend call, 1 to 65536 */
  int32_t device;           /* HIP device ordinal */
} ftcache_config;

/* Rows of tokens: element e of head h of token t is data[t * token_stride + h * head_stride + e].  data 16-byte aligned, strides
 * in elements and multiples of 8 (of 4 for 32-bit elements), so that views of a fused projection need no copy. */
typedef struct { void* data; int64_t token_stride, head_stride; } ftcache_rows;

/* Which tokens a call is about.  Sequence b has rows cu_seqlens[b] .. cu_seqlens[b + 1] of the packed tokens (cu_seqlens[0] = 0; rows
 * behind the last sequence are left as they are), which stand at the places starts[b], starts[b] + 1, .. of the sequence; place p lies in
 * page page_table[b * table_stride + p / page_size].  There are 2^31 - 16 places.  Entries of the table that no place needs may hold anything.
 * tokens / 8 + 2 * batch has to be below 2^24 (FTCACHE_EUNSUPPORTED). */
typedef struct {
  int32_t batch;             /* sequences, >= 1 */
  int32_t tokens;            /* packed rows */
  const int32_t* cu_seqlens; /* [batch + 1] */
  const int32_t* starts;     /* [batch] */
  const int32_t* page_table; /* [batch][table_stride] */
  int32_t table_width;       /* valid entries in a row of the table, 1 to table_stride */
  int64_t table_stride;
} ftcache_places;

typedef struct {
  int64_t refused_tokens;    /* tokens of append and read whose page or position does not exist */
  int64_t refused_sequences; /* sequences of attend whose length or pages do not exist */
} ftcache_report_view;

/* A context holds device memory for the states of sequences that attend divides, whatever the calls' sizes: 34 MB at head_dim 128, 17 MB at 64 (more
 * only above 2048 key / value heads).  One serves all layers of a model that run one after the other, each with a pool of its own. */
int ftcache_create(const ftcache_config* cfg, ftcache_ctx** out);
/* Copies the configuration in effect (defaults resolved). */
int ftcache_get_config(const ftcache_ctx* ctx, ftcache_config* effective);
/* Bytes of one page: kv_heads * page_size * (head_dim + 8). */
int64_t ftcache_page_bytes(const ftcache_ctx* ctx);
/* Rotates the new tokens' queries and keys by their places, writes both, and puts keys (rotated and rounded) and values into the cache.
 * rotation: [positions][rotary_dim] float32, 16-byte aligned: rotary_dim/2 cosines, then as many sines.  Products and sums of a rotation
 * are rounded one by one.  q and q_out may both be left out (data NULL), and k_out; q_out may be q, k_out may be k.  No two tokens of a call may
 * have the same place in the pool (sequences that append do not share a page); what the place holds is unspecified then. */
int ftcache_append(ftcache_ctx* ctx, void* pool, const ftcache_places* places, const float* rotation, int32_t positions,
                   const ftcache_rows* q, const ftcache_rows* k, const ftcache_rows* v, const ftcache_rows* q_out,
                   const ftcache_rows* k_out, void* hip_stream);
/* The cached keys and values of the given places, scale * c + minimum (in 32 bits) rounded to in_dtype and held to its finite numbers.  A place that nothing was appended
 * to gives what the pool holds there. */
int ftcache_read(ftcache_ctx* ctx, const void* pool, const ftcache_places* places, const ftcache_rows* k, const ftcache_rows* v,
                 void* hip_stream);
/* o[b, h] = softmax(softmax_scale * q[b, h] K^T) V over the first lengths[b] cached tokens of sequence b, one row per sequence.
 * batch * kv_heads * ceil(heads / kv_heads / 16) and some thousands more have to stay below 2^24 (FTCACHE_EUNSUPPORTED).
 * Every workgroup looks through all lengths: from some hundred sequences on the time grows with the square of the batch.
 * A length of 0 gives zeros; a 16-bit result is held to its type's finite numbers.  Codes enter the matrix products as they are and scales and minima in 32 bits; the weights are rounded
 * to bf16 once (bf16) or to two bf16 words (fp16).  Sums are held in fp32: the elements of keys and of queries, these also times softmax_scale, have to
 * stay below 2^110 and lengths[b] * max|v| below 2^127; in bf16, value scales below 2^-113 (values below about 2^-110) lose bits. */
int ftcache_attend(ftcache_ctx* ctx, const void* pool, int32_t batch, const int32_t* lengths, const int32_t* page_table,
                   int32_t table_width, int64_t table_stride, const ftcache_rows* q, const ftcache_rows* o, void* hip_stream);
/* Waits for the device, returns the counts since the last report and clears them. */
int ftcache_report(ftcache_ctx* ctx, ftcache_report_view* out);
int ftcache_destroy(ftcache_ctx* ctx);
/* Message of the last failure on this context ("" if none).  ctx may be NULL: returns the
 * message of the last failed ftcache_create of the calling thread. */
const char* ftcache_last_error(const ftcache_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* FTCACHE_H */
