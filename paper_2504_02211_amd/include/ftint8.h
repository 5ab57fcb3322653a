/*
 * ftint8.h -- C ABI of the linear layer on 8-bit integers for AMD MI355X (gfx950), part of the same shared library as ftattn.h.
 *
 * Y = X W^T as ftgemm.h has it, with the weights held in one byte each: a row of weights (an output channel) and a row of X (a token)
 * are whole numbers of -127 .. 127 times a scale of the row,
 *
 *     scale = max|x| / 127,   code = rint(x * (127 * (1 / max|x|)))            (32 bits, every step rounded; ties to even)
 *     y[t, n] = (sum over k of code_x[t, k] * code_w[n, k]) * (scale_x[t] * scale_w[n])
 *
 * The sum is exact (32-bit integers).  A row of zeros has scale 0; a row that holds an infinity or NaN has scale NaN and codes 0, which makes its
 * results NaN and no others.  Scales whose product leaves the numbers of 32 bits do so in the results: infinite, or NaN where the sum is 0.  It carries no checksums:
 * ftgemm.h is the protected form in 16 bits.
 *
 * Conventions
 *   - Every function returns FTINT8_OK (0) or a negative error code and never throws or prints; ftint8_last_error() returns the message of the last failure.
 *   - Tensors are DEVICE pointers owned by the caller.  The call leaves the current device as it was.
 *   - Codes lie as [rows][k_padded] bytes, k_padded = k rounded up to a multiple of 128, 16-byte aligned, with zeros behind column k (one operand's zeros
 *     are enough).  Codes of weights that a checkpoint brings may be used as they are, -128 among them.
 *   - ftint8_encode, ftint8_product and ftint8_forward allocate nothing and are kernel launches only on `hip_stream`: they may be recorded into a HIP graph
 *     by stream capture.  Calls on one context may not overlap in time, captured graphs of them included.
 */
#ifndef FTINT8_H
#define FTINT8_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ftint8_ctx ftint8_ctx; /* opaque, library-owned */

enum { FTINT8_F16 = 0, FTINT8_BF16 = 1, FTINT8_F32 = 2 };
enum { FTINT8_OK = 0, FTINT8_EINVAL = -1, FTINT8_EUNSUPPORTED = -2, FTINT8_EHIP = -3, FTINT8_ENOMEM = -4 };

typedef struct {
  uint32_t struct_size;  /* sizeof(ftint8_config), checked */
  int32_t n, k;          /* output and input features of the layer: any numbers from 1 on, k at most 130944 (sums of k products of codes stay below 2^31) */
  int32_t in_dtype;      /* FTINT8_F16 | FTINT8_BF16: type of x (and of weights that are encoded here) */
  int32_t out_dtype;     /* FTINT8_F32, or in_dtype */
  int32_t max_tokens;    /* most tokens of a ftint8_forward: the context holds max_tokens * (k_padded + 4) bytes for their codes and scales, and up to 8 MB */
  int32_t device;        /* HIP device ordinal */
} ftint8_config;

/* A matrix of rows: element e of row r is data[r * stride + e].  data aligned to its elements, stride in elements (any from the row's length on; rows that begin
 * at multiples of 16 bytes, and have up to 16,384 elements, are encoded two to four times as fast as others). */
typedef struct { void* data; int64_t stride; } ftint8_matrix;

int ftint8_create(const ftint8_config* cfg, ftint8_ctx** out);
/* Copies the configuration in effect (defaults resolved). */
int ftint8_get_config(const ftint8_ctx* ctx, ftint8_config* effective);
/* Bytes of a row of codes: k rounded up to a multiple of 128; negative: an error. */
int ftint8_k_padded(const ftint8_ctx* ctx);
/* Codes and scales of the rows of x, [rows, k] of in_dtype: weights once, or tokens that several layers read. */
int ftint8_encode(ftint8_ctx* ctx, const ftint8_matrix* x, int32_t rows, int8_t* codes, float* scales, void* hip_stream);
/* y [m, n] from codes and scales of m tokens, up to 2^22, and of the n channels of weights.  (More tiles of 256 x 256 than a launch has, 2^23: FTINT8_EUNSUPPORTED.) */
int ftint8_product(ftint8_ctx* ctx, const int8_t* codes_x, const float* scales_x, int32_t m, const int8_t* codes_w, const float* scales_w, const ftint8_matrix* y,
                   void* hip_stream);
/* y [m, n] from m tokens x [m, k] in 16 bits: both of the above in one call, m <= max_tokens.  The same results, bit for bit.  y and x may not overlap. */
int ftint8_forward(ftint8_ctx* ctx, const ftint8_matrix* x, int32_t m, const int8_t* codes_w, const float* scales_w, const ftint8_matrix* y, void* hip_stream);
int ftint8_destroy(ftint8_ctx* ctx);
/* Message of the last failure on this context ("" if none).  ctx may be NULL: returns the
 * message of the last failed ftint8_create of the calling thread. */
const char* ftint8_last_error(const ftint8_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* FTINT8_H */
