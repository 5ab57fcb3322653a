/*
 * ftdecay.h -- C ABI of linear attention with a decay for each head for AMD MI355X (gfx950), part of the same shared library as ftattn.h.
 *
 * Layers whose memory of a sequence is one matrix per head instead of its keys and values: for every token t of a sequence, head h and key / value head g = h / (heads / kv_heads),
 *
 *     S = exp(log_decay[h]) * S + k[t, g] v[t, g]^T          (S: head_dim x head_dim, fp32)
 *     o[t, h] = scale * q[t, h] S
 *
 * ftdecay_forward takes packed prompts (sequences of different lengths behind one another, views of a fused projection, chunks that continue an
 * earlier one), ftdecay_step one token of every sequence.  Both leave the states in a pool that the caller owns.
 *
 * What a query sees ends with its own token: later keys and values have no influence on it, not even where they are infinite or NaN.  From the token on
 * whose key or value is not finite, elements of results and states that it enters are not finite either.
 *
 * Prompts are computed in chunks of 64 tokens.  Before a product, weights q k decay^n and states are rounded to two words of 16 bits (2^-16 relative), values decayed to the end of
 * a chunk, which make the states, to three of bf16, or two of fp16: off by 2^-24 relative, or in fp16 by 2^-51 where that is more (chunks with values from 2 on in 32
 * neighbouring columns: 2^-50, and so on by octaves).  The products themselves keep 2^-24 of their largest term; elements of fp16 below 2^-14 count as 2^-14 there.  Single
 * tokens are computed in 32 bits.
 *
 * Conventions
 *   - Every function returns FTDECAY_OK (0) or a negative error code and never throws or prints; ftdecay_last_error() returns the message of the last failure.
 *   - All tensors are DEVICE pointers owned by the caller; the structures that carry them are HOST memory.  The call leaves the current device as it was.
 *   - ftdecay_forward and ftdecay_step allocate nothing and are kernel launches only on `hip_stream`: they may be recorded into a HIP graph by stream
 *     capture.  Calls on one context may not overlap in time, captured graphs of them included.
 *   - states: [n_slots][heads][head_dim of keys][head_dim of values] fp32, 16-byte aligned.  Sequence b has slot slots[b], or b where slots is NULL.  A sequence
 *     whose slot lies outside of 0 .. n_slots - 1 begins with zeros and leaves no state behind.  Each slot stands at most once in a call: where one stands
 *     twice, results and state of the sequences that name it are unspecified (nothing else is touched).
 *   - log_decay: fp32 [heads], at most 0; what is above 0, and NaN, counts as 0, -infinity forgets everything before a token.
 *   - cu begins with 0, does not fall and ends at or before total.  Bounds beyond are taken as the total: nothing out of range is read or written.  Rows of o
 *     behind the last sequence are left as they were.
 */
#ifndef FTDECAY_H
#define FTDECAY_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ftdecay_ctx ftdecay_ctx; /* opaque, library-owned */

enum { FTDECAY_F16 = 0, FTDECAY_BF16 = 1, FTDECAY_F32 = 2 };
enum { FTDECAY_OK = 0, FTDECAY_EINVAL = -1, FTDECAY_EUNSUPPORTED = -2, FTDECAY_EHIP = -3, FTDECAY_ENOMEM = -4 };

typedef struct {
  uint32_t struct_size;     /* sizeof(ftdecay_config), checked */
  int32_t heads, kv_heads;  /* heads: a multiple of kv_heads; query head h reads key / value head h / (heads / kv_heads) */
  int32_t head_dim;         /* 64 or 128 */
  int32_t in_dtype;         /* FTDECAY_F16 | FTDECAY_BF16: type of q, k, v and o */
  float scale;              /* <= 0 selects 1/sqrt(head_dim) */
  int32_t device;           /* HIP device ordinal */
} ftdecay_config;

/* Rows of tokens: element e of head h of token t is data[t * token_stride + h * head_stride + e].  data 16-byte aligned, strides
 * in elements and multiples of 8, those of tokens at most 2^24. */
typedef struct { void* data; int64_t token_stride, head_stride; } ftdecay_rows;

/* A context holds device memory for the states before and between parts of long prompts, whatever the calls' sizes: 2048 * head_dim * head_dim * 4 bytes (134 MB at 128, 34 MB at 64). */
int ftdecay_create(const ftdecay_config* cfg, ftdecay_ctx** out);
/* Copies the configuration in effect (defaults resolved). */
int ftdecay_get_config(const ftdecay_ctx* ctx, ftdecay_config* effective);
/* One pass over `batch` packed sequences: sequence b has rows cu[b] .. cu[b + 1] of q, k, v and o.  starts: tokens that sequence b had before these; 0 (or less): it begins with
 * zeros, else with its slot's state.  starts NULL: all begin with zeros.  states NULL: none are read or kept (slots and n_slots are not looked at).  o may be q, and may overlap
 * nothing else that is read. */
int ftdecay_forward(ftdecay_ctx* ctx, const ftdecay_rows* q, const ftdecay_rows* k, const ftdecay_rows* v, const ftdecay_rows* o, const float* log_decay, float* states,
                    int32_t n_slots, const int32_t* slots, const int32_t* cu, const int32_t* starts, int32_t batch, int32_t total, void* hip_stream);
/* One token of each of `batch` sequences: rows 0 .. batch - 1 of q, k, v and o; every sequence continues its slot's state. */
int ftdecay_step(ftdecay_ctx* ctx, const ftdecay_rows* q, const ftdecay_rows* k, const ftdecay_rows* v, const ftdecay_rows* o, const float* log_decay, float* states,
                 int32_t n_slots, const int32_t* slots, int32_t batch, void* hip_stream);
int ftdecay_destroy(ftdecay_ctx* ctx);
/* Message of the last failure on this context ("" if none).  ctx may be NULL: returns the
 * message of the last failed ftdecay_create of the calling thread. */
const char* ftdecay_last_error(const ftdecay_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* FTDECAY_H */
