/*
 * libasgd -- operators of a layer of experts behind k learnt centres, on one NVIDIA B200 (sm_100a), C ABI.
 *
 * A step of the K-Means worker loop (asgd.h) assigns a sample to its one nearest centre, groups the samples by
 * centre and sums them.  The operators here take the same path for a layer of experts: a token is assigned to its
 * best few experts (asgd_route), its row is brought into the experts' order in 8-bit floating point (asgd_quantize),
 * meets the expert's matrix (asgd_product), and the experts' rows are summed back into token order (asgd_combine);
 * with the gradient of each.
 *
 * General rules (those of asgd.h where they apply)
 *   - Every pointer is DEVICE memory of the current device, except the argument structures, which are HOST and are
 *     read before the call returns.  Nothing is allocated; outputs and workspaces are the caller's.  Arrays are aligned
 *     to their element (ASGD_EINVAL otherwise), and to more where it is said.
 *   - Every function returns 0 (ASGD_OK) or a negative asgd_status and enqueues its work on `stream` (a cudaStream_t,
 *     NULL = default stream); nothing is launched when it returns an error, except ASGD_ECUDA.
 *   - The functions keep no state between calls (but for the report that asgd_experts_sync takes) and may be used from
 *     several threads and streams at a time.
 *   - Sums, softmax statistics and scores are fp32 whatever the inputs' type; results do not depend on timing.
 *   - Tensors are row-major with a leading dimension (elements from one row to the next); a size of zero rows is no
 *     error: nothing is written but what does not depend on rows.
 */
#ifndef ASGD_EXPERTS_H_
#define ASGD_EXPERTS_H_

#include <stddef.h>
#include <stdint.h>

#include "asgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
enum { ASGD_F32 = 0, ASGD_BF16 = 1, ASGD_F16 = 2, ASGD_E4M3 = 3, ASGD_E5M2 = 4 };
enum { ASGD_SCORE_SOFTMAX = 0, ASGD_SCORE_SIGMOID = 1 };

#define ASGD_MAX_EXPERTS 1024
#define ASGD_MAX_EXPERT_GROUPS 32
#define ASGD_MAX_TOP_K 32
#define ASGD_PRODUCT_MAX 2147483392ll  /* 2^31 - 256: rows, columns and inner numbers of a product              */
#define ASGD_QUANTIZE_MAX 2147418112ll /* 2^31 - 65536: numbers of a row that is rounded                        */
#define ASGD_BLOCK 128 /* numbers that share a scale, along a row (and rows that do, in a 128 x 128 block) */

/*
 * Routing of tokens to experts.
 *
 * Per token with logits x[0..E):  s = softmax(x) or 1 / (1 + exp(-x));  key = s + bias.  With neither a bias nor
 * group_top = 2 the keys are the logits themselves (the same order, without a rounding).  An expert whose logit or
 * key is -inf or NaN is not available.  With groups > 1 the E experts are `groups` runs of E / groups neighbours; a
 * group scores the sum of its `group_top` largest keys (1 or 2; those that are available), and only the experts of
 * the groups_kept best groups stay.  The top_k largest keys are chosen, largest first; ties go to the lowest index,
 * among experts as among groups.  A choice's weight is scale * s, or scale * s / (sum of the chosen s + 1e-20) with
 * renormalise (the bias decides who is chosen, never the weight).  Where fewer than top_k experts are available the
 * remaining ids are -1 and their weights 0.  A NaN among a token's logits makes the softmax, and so its weights, NaN;
 * its ids stay valid.  Under softmax, logits of +inf share the probability.
 */
typedef struct asgd_route_config {
  int32_t experts;     /* E, 1..ASGD_MAX_EXPERTS                                            */
  int32_t top_k;       /* 1..min(ASGD_MAX_TOP_K, groups_kept * E / groups)                  */
  int32_t score;       /* ASGD_SCORE_*                                                      */
  int32_t groups;      /* divides E, 1..ASGD_MAX_EXPERT_GROUPS                              */
  int32_t groups_kept; /* 1..groups                                                         */
  int32_t group_top;   /* 1 or 2: keys summed for a group's score                           */
  int32_t renormalise; /* 0 or 1                                                            */
  int32_t align;       /* rows of an expert in the plan start at multiples of this, >= 1    */
  float scale;         /* factor of the weights                                             */
} asgd_route_config;

/* Bytes of workspace asgd_route() needs for T tokens (0 for few tokens; 256-byte aligned otherwise). */
int asgd_route_workspace_bytes(const asgd_route_config *cfg, int64_t T, size_t *bytes /* HOST out */);

/*
 *   logits     [T][ld >= E] of `type` ASGD_F32 / BF16 / F16          bias  [E] fp32 or NULL
 *   ids        [T][top_k] out                                        weights  [T][top_k] fp32 out
 * and the plan of the experts' order, all three or none (NULL):
 *   offsets    [E + 1] out: expert e owns the grouped rows [offsets[e], offsets[e + 1]), its assignments in ascending
 *              (token, place) order first, then rows of nothing up to the next multiple of `align`
 *   rows       [T][top_k] out: the grouped row of each assignment, -1 where the id is -1
 *   source     [source_len] out: the assignment token * top_k + place of a grouped row, -1 for rows of nothing.
 *              source_len >= T * top_k + E * (align - 1), at most 2^31 - 1
 */
int asgd_route(const asgd_route_config *cfg, int64_t T, const void *logits, int32_t type, int64_t ld, const float *bias,
               int32_t *ids, float *weights, int32_t *offsets, int32_t *rows, int32_t *source, int64_t source_len,
               void *workspace, size_t workspace_bytes, void *stream);

/* Gradient of the weights with respect to the logits, the choice held fixed:  dlogits [T][ld_out] of `type` from
 * dweights [T][top_k] fp32 and the ids of asgd_route (ids outside 0..E-1 take no part).  Uses experts, top_k, score,
 * renormalise and scale of the configuration. */
int asgd_route_grad(const asgd_route_config *cfg, int64_t T, const void *logits, int32_t type, int64_t ld,
                    const int32_t *ids, const float *dweights, void *dlogits, int64_t ld_out, void *stream);

/*
 * Rounding to 8-bit floating point with a scale for each block of 128.
 *
 * Of each block:  a = max(largest magnitude, 2^-100);  scale = a * (1 / F);  q = round(x * (F / a)), to nearest even,
 * F = 448 (E4M3) or 57344 (E5M2), every operation in fp32.  A block is 128 neighbours along a row of the result (the
 * last one of a row may be shorter) or, with `square`, 128 x 128 numbers.  An infinity or a NaN makes NaNs of its own
 * number and, with an infinity, zeros of the block's finite ones with an infinite scale.
 *
 * The rows may be gathered on the way: grouped row r is weights[source[r]] * x[source[r] / per_token] (fp32 product; no
 * factor without weights), and zeros where source[r] is negative or beyond the input.
 *
 *   q        [M][ldq]  out or NULL, its scales scale[r * scale_row + b * scale_block], b < ceil(K / 128)
 *            (with `square`: r counts blocks of 128 rows)
 *   qt       [K][ldqt] out or NULL: the transposed matrix rounded in its own blocks, 128 neighbours along M, with
 *            scales scale_t[c * scale_t_row + b * scale_t_block], b < ceil(M / 128); with `square` the transpose of q,
 *            whose scales are those of q (scale_t is not used)
 * Nothing is written between K and ldq.  ld* >= the row's length.  K above 2^25 - 512 without qt
 * and square, M above 2^23 - 128 with either, are ASGD_EUNSUPPORTED.
 */
typedef struct asgd_quantize_args {
  int64_t M, K;            /* rows and columns of the result; M <= 2^31 - 1, K <= ASGD_QUANTIZE_MAX         */
  const void *x;           /* [rows_x][ldx] of x_type, or of M rows without `source`                        */
  int64_t ldx;
  int64_t rows_x;          /* rows of x (equal to M without source)                                         */
  int32_t x_type;          /* ASGD_F32 / BF16 / F16                                                         */
  int32_t q_type;          /* ASGD_E4M3 / E5M2                                                              */
  int32_t square;          /* 0: blocks of 128 along a row, 1: 128 x 128 (no source)                        */
  int32_t per_token;       /* >= 1, see source                                                              */
  const int32_t *source;   /* [M] or NULL                                                                   */
  const float *weights;    /* [rows_x * per_token] or NULL (needs source)                                   */
  void *q;
  int64_t ldq;
  float *scale;
  int64_t scale_row, scale_block;
  void *qt;
  int64_t ldqt;
  float *scale_t;
  int64_t scale_t_row, scale_t_block;
} asgd_quantize_args;

int asgd_quantize(const asgd_quantize_args *args, void *stream);

/*
 * Product of 8-bit matrices with block scales:
 *   C[m][n] = sum over blocks b of 128 along K of  sA(m, b) * sB(n, b) * sum_{k in b} A[m][k] * B[n][k]
 * The inner sums are tensor-core sums in fp32, the outer one is fp32; C is rounded once.
 *
 *   sA(m, b) = a_scale[m * a_scale_row + b * a_scale_block];  sB the same with n, or with n / 128 when b_square is set.
 *
 * groups = 0: one product.  groups > 0, over the rows (inner = 0): row m belongs to the group g with
 * offsets[g] <= m < offsets[g + 1] and meets B_g = B + g * b_group, with scales b_scale + g * b_scale_group; rows
 * outside all groups are not written.  groups > 0, inner = 1: A is [M][K] and B [N][K] once, and C_g = C + g * c_group
 * sums over k in [offsets[g], offsets[g + 1]) alone (zeros for an empty group).  Offsets are ascending; bounds beyond
 * the matrix are cut off.  With inner = 1 every bound has to be a multiple of 128 or K itself; a group that breaks
 * this is written as NaN and reported by asgd_experts_sync as ASGD_EINVAL.
 *
 * A, B: E4M3 or E5M2 (each its own), 16-byte aligned, leading dimensions and b_group multiples of 16.  C: fp32, bf16
 * or fp16, aligned to its element.  ASGD_EINVAL otherwise.
 */
typedef struct asgd_product_args {
  int64_t M, N, K;         /* each <= ASGD_PRODUCT_MAX (ASGD_EUNSUPPORTED above) */
  const void *a;
  int64_t lda;
  const float *a_scale;
  int64_t a_scale_row, a_scale_block;
  const void *b;
  int64_t ldb, b_group;
  const float *b_scale;
  int64_t b_scale_row, b_scale_block, b_scale_group;
  void *c;
  int64_t ldc, c_group;
  const int32_t *offsets;  /* [groups + 1] or NULL */
  int32_t groups;          /* 0..ASGD_MAX_EXPERTS */
  int32_t inner;
  int32_t a_type, b_type, c_type;
  int32_t b_square;
} asgd_product_args;

int asgd_product(const asgd_product_args *args, void *stream);

/*
 * Rows of the experts back into token order:  y[t] = sum_j weights[t][j] * z[rows[t][j]]  (fp32 sums in ascending j;
 * factors 1 without weights; rows outside 0..R-1 take no part), y and z of `type`.
 * Gradient: dz[rows[t][j]] = weights[t][j] * dy[t] (dz may be NULL), dweights[t][j] = <dy[t], z[rows[t][j]]> (may be
 * NULL), 0 where the row takes no part; the rows of dz whose source (see asgd_route; may be NULL) is negative become 0.
 * D above 2^22 may be ASGD_EUNSUPPORTED.
 */
int asgd_combine(int64_t T, int64_t D, int32_t top_k, const void *z, int32_t type, int64_t R, int64_t ldz,
                 const int32_t *rows, const float *weights, void *y, int64_t ldy, void *stream);
int asgd_combine_grad(int64_t T, int64_t D, int32_t top_k, const void *dy, int32_t type, int64_t ld_dy, const void *z,
                      int64_t R, int64_t ldz, const int32_t *rows, const float *weights, const int32_t *source, void *dz,
                      int64_t ld_dz, float *dweights, void *stream);

/* Wait for the stream and return what asgd_product calls on this device (and those of asgd_product4, asgd_fp4.h, and
 * asgd_expert_layer, asgd_expert_layer.h) have reported since the last asgd_experts_sync: ASGD_OK, ASGD_EINVAL (offsets, see above) or ASGD_ETIMEOUT (a bounded wait on the kernel's own copies or products ran
 * out; the outputs of that call are not to be used); of several the last named.  This is the one state between calls:
 * there is one report per device, shared by all of its streams, and the call that takes it clears it (no report that comes
 * meanwhile is lost).  With several streams in use, wait for all of them, then call this once for all. */
int asgd_experts_sync(void *stream);
/* Failure drill of these functions' bounded waits, as asgd_set_wait_drill: later launches of this process give a wait up
 * after wait_limit polls (copies and products in flight end all the same before a kernel leaves), and with withhold = 1 the first copy of every block is announced but never issued.
 * Defaults 2^22 and 0.  ASGD_EINVAL for wait_limit = 0. */
int asgd_product_set_wait_drill(uint32_t wait_limit, int32_t withhold);

#ifdef __cplusplus
}
#endif
#endif /* ASGD_EXPERTS_H_ */
