/*
 * ftprompt.h -- C ABI of attention over packed prompts for AMD MI355X (gfx950), part of the same shared library as ftattn.h.
 *
 * The pass of ftattn.h with its checks off, for what a decoder's prefill brings: sequences of different lengths packed
 * behind one another, fewer key / value heads than query heads, tensors that are views of a fused projection, and queries whose
 * keys begin before them (a chunk of a prompt over its cached prefix).  Sequence b has query rows cu_q[b] .. cu_q[b + 1] and key rows
 * cu_k[b] .. cu_k[b + 1]; the last query stands at the last key, and a query sees the keys up to its own place:
 *
 *     o[i, h] = sum over j <= nk - nq + i of softmax_j(softmax_scale * q[i, h] . k[j, h / (heads / kv_heads)]) v[j, same head]
 *
 * A query that sees no key, or only scores of -infinity, gives zeros.  Keys and values behind a query's place have no influence
 * on it, not even where they are infinite or NaN.  Where a query sees values that are infinite or NaN, their element of its result is the sum of
 * them, however small their weights.  It carries no checksums: ftattn.h is the protected form for batches of one length.
 *
 * Conventions
 *   - Every function returns FTPROMPT_OK (0) or a negative error code and never throws or prints; ftprompt_last_error()
 *     returns the message of the last failure.
 *   - q, k, v, o, cu_q, cu_k are DEVICE pointers owned by the caller; the structures that carry them are HOST memory.  The call leaves
 *     the current device as it was.
 *   - ftprompt_forward allocates nothing and is kernel launches only on `hip_stream`: it may be recorded into a HIP graph by stream
 *     capture.  Calls on one context may not overlap in time, captured graphs of them included.
 *   - cu_q and cu_k begin with 0, do not fall and end at or before total_q and total_k.  Bounds beyond those are taken as the totals: nothing
 *     out of range is read or written.  Rows of o behind the last sequence are left as they were.
 */
#ifndef FTPROMPT_H
#define FTPROMPT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ftprompt_ctx ftprompt_ctx; /* opaque, library-owned */

enum { FTPROMPT_F16 = 0, FTPROMPT_BF16 = 1, FTPROMPT_F32 = 2 };
enum { FTPROMPT_OK = 0, FTPROMPT_EINVAL = -1, FTPROMPT_EUNSUPPORTED = -2, FTPROMPT_EHIP = -3, FTPROMPT_ENOMEM = -4 };

typedef struct {
  uint32_t struct_size;     /* sizeof(ftprompt_config), checked */
  int32_t heads, kv_heads;  /* heads: a multiple of kv_heads; query head h reads key / value head h / (heads / kv_heads) */
  int32_t head_dim;         /* 64 or 128 */
  int32_t in_dtype;         /* FTPROMPT_F16 | FTPROMPT_BF16: the products run on the MFMA of that type with fp32 accumulation;
                               weights are rounded to it before they meet the values.  Sums of keys' weights of at most 1 (bf16; 2^14
                               in fp16) times values are held in fp32: in bf16 keys * max|v| has to stay below its largest number */
  int32_t out_dtype;        /* FTPROMPT_F32, or in_dtype */
  float softmax_scale;      /* <= 0 selects 1/sqrt(head_dim) */
  int32_t device;           /* HIP device ordinal */
} ftprompt_config;

/* Rows of tokens: element e of head h of token t is data[t * token_stride + h * head_stride + e].  data 16-byte aligned, strides
 * in elements and multiples of 8 (of 4 for 32-bit elements), at most 2^24. */
typedef struct { void* data; int64_t token_stride, head_stride; } ftprompt_rows;

/* A context holds device memory for the states of row tiles that are divided by their keys, whatever the calls' sizes: 69 MB at head_dim 128, 36 MB
 * at 64.  One serves all layers of a model that run one after the other. */
int ftprompt_create(const ftprompt_config* cfg, ftprompt_ctx** out);
/* Copies the configuration in effect (defaults resolved). */
int ftprompt_get_config(const ftprompt_ctx* ctx, ftprompt_config* effective);
/* One pass over `batch` sequences.  cu_k may be cu_q: prompts that begin with their first key.  o may be q.  Calls of more than 64 sequences divide no
 * row tile by its keys: a few queries over long prefixes on one or two key heads are faster in calls of 64.  total_q * heads / 128 + batch * kv_heads and some
 * hundreds more have to stay below 2^24 (FTPROMPT_EUNSUPPORTED). */
int ftprompt_forward(ftprompt_ctx* ctx, const ftprompt_rows* q, const ftprompt_rows* k, const ftprompt_rows* v, const ftprompt_rows* o,
                     const int32_t* cu_q, const int32_t* cu_k, int32_t batch, int32_t total_q, int32_t total_k, void* hip_stream);
int ftprompt_destroy(ftprompt_ctx* ctx);
/* Message of the last failure on this context ("" if none).  ctx may be NULL: returns the
 * message of the last failed ftprompt_create of the calling thread. */
const char* ftprompt_last_error(const ftprompt_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* FTPROMPT_H */
