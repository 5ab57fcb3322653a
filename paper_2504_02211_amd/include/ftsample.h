/*
 * ftsample.h -- C ABI of the choice of the next token for AMD MI355X (gfx950), part of the same shared library as ftattn.h.
 *
 * What ends a decoding step: from the logits x of a row and a given random number u, with the row's own temperature T, top_k, top_p and min_p,
 *
 *     w[i] = exp((x[i] - max x) / T)
 *     top_k: the top_k largest are kept;
 *     top_p: of those, in falling order, the ones before which the sum of weights is below top_p times the sum of all of them;
 *     min_p: of those, the ones with w >= min_p;
 *     the token is the first, in the order of the vocabulary, at which the sum of the kept weights exceeds u times the sum of all of them.
 *
 * Of equal logits the one of lower index is the larger one, and the largest is always kept.  Logits of -infinity, and NaN, are never chosen; a row that has
 * nothing else gives token -1 and probability 0.  Where the largest logit is +infinity, those that are so share the row equally.  T <= 0 gives the largest logit.
 * A row's result depends on that row alone, and is the same in every call: weights are computed in 64 bits and summed as whole multiples of 2^-50 (2^-62 * vocab for vocabularies above 4096,
 * vocab rounded up to a power of two), so that no sum depends on its order.
 *
 * Conventions
 *   - Every function returns FTSAMPLE_OK (0) or a negative error code and never throws or prints; ftsample_last_error() returns the message of the last failure.
 *   - All arrays are DEVICE pointers owned by the caller.  The call leaves the current device as it was.
 *   - ftsample_choose allocates nothing and is kernel launches only on `hip_stream`: it may be recorded into a HIP graph by stream capture.  Calls on one context may
 *     not overlap in time, captured graphs of them included.
 */
#ifndef FTSAMPLE_H
#define FTSAMPLE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ftsample_ctx ftsample_ctx; /* opaque, library-owned */

enum { FTSAMPLE_F16 = 0, FTSAMPLE_BF16 = 1, FTSAMPLE_F32 = 2 };
enum { FTSAMPLE_OK = 0, FTSAMPLE_EINVAL = -1, FTSAMPLE_EUNSUPPORTED = -2, FTSAMPLE_EHIP = -3, FTSAMPLE_ENOMEM = -4 };

typedef struct {
  uint32_t struct_size;  /* sizeof(ftsample_config), checked */
  int32_t vocab;         /* logits of a row, 1 .. 2^20 */
  int32_t max_rows;      /* most rows of a call, 1 .. 65536 */
  int32_t in_dtype;      /* type of the logits */
  int32_t device;        /* HIP device ordinal */
} ftsample_config;

/* The rules of every row: arrays of `rows` elements, or NULL for none. */
typedef struct {
  const float* temperature;  /* NULL: 1 */
  const int32_t* top_k;      /* 0 or less: no limit */
  const float* top_p;        /* 1 or more, or NaN: no limit; 0 or less: the largest alone */
  const float* min_p;        /* relative to the largest weight; 0 or less, or NaN: no limit; above 1: as 1 */
} ftsample_rules;

int ftsample_create(const ftsample_config* cfg, ftsample_ctx** out);
/* Copies the configuration in effect (defaults resolved). */
int ftsample_get_config(const ftsample_ctx* ctx, ftsample_config* effective);
/* tokens [rows] (and probability [rows], or NULL: the chosen token's share of the kept weights) from logits [rows][vocab], rows row_stride elements apart, and one random number of
 * [0, 1) per row (what lies outside, or is NaN, is taken as the nearer end, NaN as 0).  A temperature of NaN counts as 1. */
int ftsample_choose(ftsample_ctx* ctx, const void* logits, int64_t row_stride, int32_t rows, const float* uniform, const ftsample_rules* rules, int32_t* tokens,
                    float* probability, void* hip_stream);
int ftsample_destroy(ftsample_ctx* ctx);
/* Message of the last failure on this context ("" if none).  ctx may be NULL: returns the
 * message of the last failed ftsample_create of the calling thread. */
const char* ftsample_last_error(const ftsample_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* FTSAMPLE_H */
