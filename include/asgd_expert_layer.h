/*
 * libasgd -- a whole layer of experts for a few tokens, on one NVIDIA B200 (sm_100a), C ABI.
 *
 * What asgd_route, asgd_quantize, asgd_product, an activation, asgd_quantize, asgd_product and asgd_combine
 * (asgd_experts.h) do one after another for a batch, in one kernel for the few tokens of a serving step.  The general rules are those
 * of asgd_experts.h.
 */
#ifndef ASGD_EXPERT_LAYER_H_
#define ASGD_EXPERT_LAYER_H_

#include <stddef.h>
#include <stdint.h>

#include "asgd_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ASGD_ACT_RELU2 = 0 /* max(u, 0)^2 */, ASGD_ACT_SILU = 1 /* u / (1 + exp(-u)) */ };

#define ASGD_LAYER_MAX_TOKENS 128       /* T                                                                  */
#define ASGD_LAYER_MAX_ASSIGNMENTS 1024 /* T * top_k                                                          */
#define ASGD_LAYER_MAX_WIDTH 65536      /* d and the rows of W1                                               */

/*
 * For each token t with row x of X:
 *   logits   as given, or ((x . router[e]) - shift[e]) * temperature, fp32 (shift: 0 where there is none)
 *   e_j, w_j the choice and the weights that asgd_route gives for these logits, bit by bit
 *   xq       x rounded to E4M3 in blocks of 128 (asgd_quantize)
 *   u        = W1[e_j] xq                          h or, gated, 2 h numbers
 *   a        = act(u), or act(u[i]) * u[h + i]     h numbers
 *   aq       a rounded to E4M3 in blocks of 128
 *   y        = sum_j w_j W2[e_j] aq                d numbers, over the choices in their order (those with an expert)
 * A token without an expert has y = 0; but NaN where the logits are made here and x or one of its logits is not a number, or x infinite.
 * Everything between is fp32; the products' sums are those of asgd_product, K block by K block of 128, in stretches that depend
 * on the sizes and the loads of the experts alone; y is rounded once.
 *
 * W1 [E][rows][ldw1], W2 [E][d][ldw2]: E4M3 or E5M2 with scales of 128 x 128 blocks (asgd_quantize, square), 16-byte aligned;
 * ld* and the strides from expert to expert are multiples of 16.
 */
typedef struct asgd_expert_layer_args {
  int64_t T, d, h;         /* tokens, width of a token, hidden numbers of an expert; d, h >= 1              */
  const void *x;           /* [T][ldx] of `type`                                                            */
  int64_t ldx;
  void *y;                 /* [T][ldy] of `type` out                                                        */
  int64_t ldy;
  const void *logits;      /* [T][ld_logits] of logits_type, or NULL with a router                          */
  int64_t ld_logits;
  const void *router;      /* [E][ld_router] of router_type, or NULL with logits                            */
  int64_t ld_router;
  const float *shift;      /* [E] or NULL (needs a router)                                                  */
  const float *bias;       /* [E] or NULL: takes part in the choice alone (asgd_route)                      */
  const void *w1;
  int64_t ldw1, w1_group;  /* bytes from row to row and from expert to expert                               */
  const float *w1_scale;   /* [e * w1_scale_group + (row / 128) * w1_scale_row + (column / 128) * w1_scale_block] */
  int64_t w1_scale_row, w1_scale_block, w1_scale_group;
  const void *w2;
  int64_t ldw2, w2_group;
  const float *w2_scale;
  int64_t w2_scale_row, w2_scale_block, w2_scale_group;
  int32_t *ids;            /* [T][top_k] out or NULL                                                        */
  float *weights;          /* [T][top_k] out or NULL                                                        */
  int32_t type;            /* ASGD_F32 / BF16 / F16                                                         */
  int32_t logits_type, router_type;
  int32_t w1_type, w2_type; /* ASGD_E4M3 / E5M2                                                             */
  int32_t gated;           /* 0: W1 has h rows, 1: 2 h                                                      */
  int32_t activation;      /* ASGD_ACT_*                                                                    */
  float temperature;
} asgd_expert_layer_args;

/* Bytes of workspace that asgd_expert_layer() needs (256-byte aligned), for any pointers and loads.  `cfg` is asgd_route's;
 * its align has no part here. */
int asgd_expert_layer_workspace_bytes(const asgd_route_config *cfg, const asgd_expert_layer_args *args, size_t *bytes /* HOST out */);

/* The kernel takes all SMs at once (a cooperative launch).  ASGD_EUNSUPPORTED beyond the limits above, or where the layer
 * is too wide for 32-bit numbers of its K blocks.  A bounded wait that runs out is reported by asgd_experts_sync;
 * asgd_product_set_wait_drill covers this call. */
int asgd_expert_layer(const asgd_route_config *cfg, const asgd_expert_layer_args *args, void *workspace,
                      size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ASGD_EXPERT_LAYER_H_ */
