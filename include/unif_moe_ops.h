/*
 * unif_moe_ops.h - operators around a UniF-MoE layer in a training or serving
 * step, exported by the same library as unif_moe.h and under the same
 * conventions: device pointers owned by the caller, nothing allocated, no
 * state kept between calls, asynchronous on `stream`, arguments validated on
 * the host before any HIP call, row-major layouts, bf16 as 16-bit words
 * rounded to nearest even.
 *
 *   unif_moe_residual_forward / _backward   the end of a block's branch joined
 *       with the residual stream (norm behind the branch, gate, residual
 *       scale) and the norm in front of the next block, in one pass
 *   unif_moe_balance_loss   balance loss of the residual experts over a
 *       routing record, per-expert counts, and the loss's gradient
 *
 * One training step of a block: h = N_in(x) (residual_forward without a
 * branch), unif_moe_layer_forward on h, residual_forward on its output (which
 * also forms the next block's h); back: residual_backward, then
 * unif_moe_layer_backward on df, unif_moe_balance_loss and
 * unif_moe_diversity_loss adding to the layer's gradients, and the next
 * residual_backward with the layer's dX as dh.
 */
#ifndef UNIF_MOE_OPS_H
#define UNIF_MOE_OPS_H

#include "unif_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Row norms over the d features of a token, with optional shift beta:
 *   LAYER  N(u) = (u - mean(u)) / sqrt(var(u) + eps) * gamma + beta (biased var)
 *   RMS    N(u) = u / sqrt(mean(u^2) + eps) * gamma + beta
 *   NONE   N(u) = u */
#define UNIF_ROWNORM_NONE  0
#define UNIF_ROWNORM_LAYER 1
#define UNIF_ROWNORM_RMS   2

/* Narrowest and widest rows of the residual operators. */
#define UNIF_RESIDUAL_MIN_D 4
#define UNIF_RESIDUAL_MAX_D 8192

/* The join of a block's branch f with the residual stream x, and the norm in
 * front of the next block, per token:
 *   v = residual_scale * x + gate * N_out(f),   y = v,   h = N_in(v). */
typedef struct unif_moe_residual {
    int32_t n_tokens;        /* N >= 0 rows                                          */
    int32_t d_model;         /* d in [UNIF_RESIDUAL_MIN_D, UNIF_RESIDUAL_MAX_D]      */
    int32_t dtype;           /* UNIF_F32 or UNIF_BF16: f, h and df (what the layer
                                takes and returns)                                   */
    int32_t stream_dtype;    /* x, y, dy and dx: UNIF_F32, or UNIF_BF16 where dtype
                                is UNIF_BF16                                         */
    int32_t out_norm;        /* UNIF_ROWNORM_* of N_out, behind the branch           */
    int32_t in_norm;         /* UNIF_ROWNORM_* of N_in, in front of the next block   */
    int32_t tokens_per_gate; /* 0: one gate row for every token; R > 0: a gate row
                                per R consecutive tokens (one sequence or image),
                                ceil(N / R) rows. Unused without a gate              */
    float   out_eps, in_eps; /* eps >= FLT_MIN, finite (unused for NONE)             */
    float   residual_scale;  /* finite; a constant, without a gradient               */
    const float* out_gamma;  /* [d] fp32 device array; NULL exactly for NONE         */
    const float* out_beta;   /* [d] or NULL (no shift); NULL for NONE                */
    const float* in_gamma;   /* as out_gamma, out_beta, for N_in                     */
    const float* in_beta;
    const float* gate;       /* [1 or ceil(N / R), d] fp32, or NULL (gate 1)         */
} unif_moe_residual;

/* Forward of the join.
 *   x      [N, d] stream_dtype, or NULL: no residual (v = gate * N_out(f))
 *   f      [N, d] dtype, or NULL: no branch (v = residual_scale * x; out_norm
 *          must be NONE and gate NULL). x or f must be given
 *   valid  [N] uint8, nonzero = real token; NULL means all valid. Padded
 *          tokens are skipped: their rows of y and h are zero, whatever x, f and
 *          parameters hold there (a gate row that only padded tokens have)
 *   y      [N, d] stream_dtype, or NULL: not written. May be x itself
 *   h      [N, d] dtype, or NULL: not written; needs in_norm other than NONE
 * Other overlaps of outputs with inputs or each other are rejected. Tensors
 * are aligned to their elements; any d (rows need no padding).
 * Precision: sums, statistics and the row itself in fp32; y and h are each
 * rounded once (h is formed from the unrounded v). Values beyond about 1e18
 * in magnitude overflow the statistics.
 * Errors: UNIF_EINVAL, UNIF_EUNSUPPORTED (d out of range) before any
 * launch; UNIF_EDEVICE if a launch fails. */
int32_t unif_moe_residual_forward(const unif_moe_residual* res, const void* x, const void* f,
                                  const uint8_t* valid, void* y, void* h, void* stream);

/* Parameter gradients of the join (fp32 device arrays of the parameters'
 * shapes, written; NULL: not wanted). Those of parameters that `res` lacks
 * must be NULL. */
typedef struct unif_moe_residual_grads {
    float* out_gamma;
    float* out_beta;
    float* in_gamma;
    float* in_beta;
    float* gate;
} unif_moe_residual_grads;

/* Workspace needed by unif_moe_residual_backward (bytes). Host only. */
int32_t unif_moe_residual_backward_workspace_size(const unif_moe_residual* res, size_t* bytes);

/* Backward of the join: with the gradients dy of y and dh of h,
 *   D = dy + (d h / d v)^T dh      (gradient of v)
 *   dx = residual_scale * D,  df = (d v / d f)^T D,  and the parameters'.
 *   y      [N, d] stream_dtype: the forward's y (v is taken from it); NULL
 *          exactly where dh is NULL
 *   f      [N, d] dtype: the forward's branch; needed for df and the gradients
 *          of gate and N_out unless out_norm is NONE and only df is wanted
 *   valid  as in the forward: padded tokens get dx = df = 0 and add nothing to
 *          any gradient, whatever the inputs and parameters hold there; the
 *          gradient of a gate row that only padded tokens have is 0
 *   dy     [N, d] stream_dtype, or NULL (0)
 *   dh     [N, d] dh_dtype, or NULL (0); needs in_norm other than NONE. dy or
 *          dh must be given
 *   dh_dtype  UNIF_F32 (what unif_moe_layer_backward writes) or the layer's
 *   dx     [N, d] stream_dtype, or NULL: not wanted. May be dy itself
 *   df     [N, d] dtype, or NULL: not wanted
 *   grads  or NULL: none wanted
 * Other overlaps of outputs with inputs or each other are rejected.
 * Sums in fp32 (a parameter's over the tokens: fp32 within a workgroup's
 * tokens, then fp64), every one in a fixed order: repeated calls give the same
 * bits. Errors: as the forward, and UNIF_EWORKSPACE. */
int32_t unif_moe_residual_backward(const unif_moe_residual* res, const void* y, const void* f,
                                   const uint8_t* valid, const void* dy, const void* dh, int32_t dh_dtype,
                                   void* dx, void* df, const unif_moe_residual_grads* grads, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* Narrowest layers whose balance gradients are formed. */
#define UNIF_BALANCE_MIN_D 8

/* What an expert's load counts. */
#define UNIF_BALANCE_TOKENS 0 /* tokens that run the expert                          */
#define UNIF_BALANCE_BLOCKS 1 /* blocks those tokens run of it: B - b each           */

typedef struct unif_moe_balance {
    int32_t tokens_per_group; /* 0: all tokens in one group; R > 0: a group per R
                                 consecutive tokens (a sequence), G = ceil(N / R)    */
    int32_t unit;             /* UNIF_BALANCE_*                                      */
    float   weight;           /* lambda, finite: factor of the gradients             */
} unif_moe_balance;

/* Workspace needed by unif_moe_balance_loss (bytes). Host only. */
int32_t unif_moe_balance_loss_workspace_size(const unif_moe_config* cfg, const unif_moe_balance* bal,
                                             size_t* bytes);

/* Balance loss of the residual experts over the routing record of this layer
 * and these tokens (unif_moe_route or a forward). For each group s with n_s
 * valid tokens, c_sj the load of expert j (over the tokens whose first n_res
 * experts hold j) and p_tj the softmax affinity:
 *   L_s = K sum_j (c_sj / sum_m c_sm) (1 / n_s) sum_{t in s} p_tj
 *   *loss = L = (1 / G) sum_s L_s
 * (1 where loads and affinities are uniform; a group without a valid token or
 * without any load counts as 0). The loads are piecewise constant and held
 * fixed; the gradient flows through the affinities to W_1..W_K and x:
 *   d L / d l_tj = (K / (G n_s sum_m c_sm)) p_tj (c_sj - sum_m p_tm c_sm)
 *   dX        = [dX_in +]        weight * sum_j (d L / d l_tj) W_j
 *   dW_router = [dW_router_in +] weight * sum_t (d L / d l_tj) x_t  (row 0: + 0)
 *   record     of cfg's N and K; n_shared is read for UNIF_BALANCE_BLOCKS.
 *              Expert ids outside 1..K are ignored
 *   valid      [N] uint8 or NULL, as the record was made with
 *   X          [N, d] cfg->dtype (needed with dW_router)
 *   W_router   [K+1, d] fp32 (needed with dX)
 *   loss       [1] fp32, written
 *   counts     [G, K+1] int64, written, or NULL: column j the load c_sj, column
 *              0 the shared expert's (valid tokens, or their blocks sum b)
 *   dX_in      [N, d] fp32 or NULL (0); may be dX itself (added in place)
 *   dX         [N, d] fp32, or NULL: not wanted. Padded tokens get dX_in's rows,
 *              whatever W_router holds
 *   dW_router_in, dW_router   [K+1, d] fp32, likewise
 * A training step calls it after unif_moe_layer_backward with the layer's
 * gradients in place. cfg is validated as for the layer; N, d, K, B and dtype
 * are read (d <= 2^20). Other overlaps of outputs with inputs or each other are
 * rejected.
 * Precision: p, the loads' shares and the gradients in fp32, sums over tokens
 * in fp32 within a workgroup's tokens and in fp64 past that, in a fixed order:
 * repeated calls give the same bits.
 * Errors: UNIF_EINVAL, UNIF_EWORKSPACE, UNIF_EUNSUPPORTED (also gradients of d <
 * UNIF_BALANCE_MIN_D) before any launch; UNIF_EDEVICE if a launch fails. */
int32_t unif_moe_balance_loss(const unif_moe_config* cfg, const unif_moe_balance* bal,
                              const unif_moe_routing* record, const uint8_t* valid, const void* X,
                              const float* W_router, float* loss, int64_t* counts, const float* dX_in,
                              float* dX, const float* dW_router_in, float* dW_router, void* workspace,
                              size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* UNIF_MOE_OPS_H */
