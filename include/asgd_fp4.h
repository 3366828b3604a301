/*
 * libasgd -- microscaled 4-bit operands and their products, on one NVIDIA B200 (sm_100a), C ABI.
 *
 * The 4-bit siblings of the 8-bit operands and products of asgd_experts.h: half the bytes of the weights, which are what a
 * serving step of few tokens waits for, and twice the tensor cores' rate.  Forward form: gradients have a range that 4 bits
 * do not reach, and stay with the 8-bit operators (the master weights are the caller's either way).
 *
 * The general rules are those of asgd_experts.h.
 *
 * The format.  A number is E2M1: 0, 1/2, 1, 3/2, 2, 3, 4 or 6 and a sign; 32 neighbours along a row (the last block of a row
 * may be shorter) share a power of two, stored as a byte c that stands for 2^(c - 127), 255 for NaN.  A byte holds two numbers, that of
 * the lower column in its lower four bits; where a row's length is odd the upper four bits of its last byte are 0.
 */
#ifndef ASGD_FP4_H_
#define ASGD_FP4_H_

#include <stddef.h>
#include <stdint.h>

#include "asgd_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ASGD_BLOCK4 32

/*
 * Rounding to 4 bits.  Of each block:  a = max(largest magnitude, 2^-100);  s = the smallest power of two with a <= 6 s;
 * q = x / s rounded to nearest, ties to the number with an even last bit (nothing is clipped).  A block with an infinity or a
 * NaN has the scale NaN and zeros.  The rows may be gathered and weighted on the way, as asgd_quantize does it.
 */
typedef struct asgd_quantize4_args {
  int64_t M, K;            /* rows and columns of the result; M <= 2^31 - 1, above K = 2^25 - 519
                              ASGD_EUNSUPPORTED (so for asgd_dequantize4)                                   */
  const void *x;           /* [rows_x][ldx] of x_type, or of M rows without `source`                        */
  int64_t ldx;
  int64_t rows_x;          /* rows of x (equal to M without source)                                         */
  int32_t x_type;          /* ASGD_F32 / BF16 / F16                                                         */
  int32_t per_token;       /* >= 1, see asgd_quantize                                                       */
  const int32_t *source;   /* [M] or NULL                                                                   */
  const float *weights;    /* [rows_x * per_token] or NULL (needs source)                                   */
  void *q;                 /* [M][ldq bytes], ldq >= ceil(K / 2)                                            */
  int64_t ldq;
  void *scale;             /* [M][scale_row bytes], scale_row >= ceil(K / 32)                               */
  int64_t scale_row;
} asgd_quantize4_args;

int asgd_quantize4(const asgd_quantize4_args *args, void *stream);

/* What 4-bit rows stand for:  out [M][ld_out] of `type` from q [M][ldq bytes] and scale [M][scale_row bytes]; each number
 * times its power of two, rounded once (fp32 holds all but those beyond its range). */
int asgd_dequantize4(int64_t M, int64_t K, const void *q, int64_t ldq, const void *scale, int64_t scale_row, void *out,
                     int32_t type, int64_t ld_out, void *stream);

/*
 * Product of 4-bit matrices:  C[m][n] = sum over k of A[m][k] * B[n][k] of what the numbers stand for; sums on the tensor
 * cores in fp32, C rounded once.
 *
 * groups = 0: one product.  groups > 0: row m belongs to the group g with offsets[g] <= m < offsets[g + 1] and meets
 * B_g = B + g * b_group with scales b_scale + g * b_scale_group; rows outside all groups are not written.  Offsets are
 * ascending; bounds beyond the matrix are cut off.
 *
 * A, B and their scales are 16-byte aligned; lda, ldb, b_group, a_scale_row, b_scale_row and b_scale_group (bytes) are multiples of 16.
 * C: fp32, bf16 or fp16, aligned to its element.  ASGD_EINVAL otherwise.  A bounded wait that runs out is reported by
 * asgd_experts_sync; asgd_product_set_wait_drill covers this call.
 */
typedef struct asgd_product4_args {
  int64_t M, N, K;         /* numbers, each <= ASGD_PRODUCT_MAX (ASGD_EUNSUPPORTED above) */
  const void *a;
  int64_t lda;             /* bytes, >= ceil(K / 2) */
  const void *a_scale;
  int64_t a_scale_row;     /* bytes, >= ceil(K / 32) */
  const void *b;
  int64_t ldb, b_group;
  const void *b_scale;
  int64_t b_scale_row, b_scale_group;
  void *c;
  int64_t ldc;             /* elements */
  const int32_t *offsets;  /* [groups + 1] or NULL */
  int32_t groups;          /* 0..ASGD_MAX_EXPERTS */
  int32_t c_type;
} asgd_product4_args;

int asgd_product4(const asgd_product4_args *args, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ASGD_FP4_H_ */
