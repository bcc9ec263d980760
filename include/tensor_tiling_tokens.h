/* tensor_tiling_tokens.h - what a chain of layers needs around it to train a token model, under the conventions of
 * tensor_tiling.h (shards, tilings, statuses, streams, workspaces): the embedding in front of the chain and its table's
 * gradient, the clipped policy loss behind it and its gradient, and activations that are kept in 8 bits between the
 * forward and the backward pass.
 *
 * Per-token values (token numbers, log probabilities, weights) are whole arrays, one entry per token, dense and in one
 * device buffer whatever the tilings are: they are as small as a row of pointers.  Token numbers are TT_I32 or TT_I64.
 * Shards, and buffers that a call writes, must not overlap any other buffer given to it.
 *
 * Calls with no tokens, rows or columns return TT_OK and write nothing, but for tt_policy_loss's loss (0), a table gradient
 * without tokens (zeros), and log probabilities of an empty vocabulary (0); shards of a tensor without values may be NULL.
 * (tt_fc_backward_packed takes a batch of 1 and more, as tt_fc_backward does.)  Errors as in tensor_tiling.h: TT_EINVAL (NULL,
 * unknown type or letter, k out of range, negative or misaligned), TT_EINFEASIBLE (uneven cut), TT_EUNSUPPORTED (2^31 tokens, rows,
 * columns or vocabulary entries and more; 2^30 numbers of an embedding; 2^22 tokens of a loss), TT_EWORKSPACE, TT_EDEVICE. */
#ifndef TENSOR_TILING_TOKENS_H
#define TENSOR_TILING_TOKENS_H

#include "tensor_tiling.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TT_I32 = 2, TT_I64 = 3 }; /* types of token numbers */
/* tt_kernel_record.kernel of these calls' launches: rows = d0, columns = d1, element bytes = d2 */
enum { TT_K_EMBED = 12, TT_K_EMBED_GRAD = 13, TT_K_LOSS = 14, TT_K_PACK = 15, TT_K_UNPACK = 16 };

/* --------------------------------------------------------------- embedding */

/* X[t] = scale * W[ids[t]] for every token t (one fp32 product per value, rounded to dtype once); a row of zeros where
 * ids[t] lies outside [0, vocab) (padding).  W: vocab x width under tW;  X: tokens x width under tX, replicas written
 * once each;  dtype of both TT_F32 | TT_BF16. */
tt_status tt_embed_forward(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, tt_tiling tW, tt_tiling tX,
                           int id_dtype, const void *ids, float scale, const void *const *W, void *const *X, void *stream);

/* dW[v] = scale * sum of dX[t] over the tokens t with ids[t] = v (zeros where there is none), every row written.  The
 * sums are fp32 and run over the tokens sorted by number, in an order that depends on ids alone, so equal calls give equal
 * bits; one rounding to dtype.  dX: tokens x width under tdX;  dW: vocab x width under tdW.
 * Workspace: device memory, 256-byte aligned, at least tt_embed_workspace_bytes (may be NULL if 0); nothing in it needs
 * clearing.  What is enough for so many tokens is enough for fewer. */
tt_status tt_embed_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, tt_tiling tdX, tt_tiling tdW,
                                   size_t *bytes);
tt_status tt_embed_backward(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, tt_tiling tdX, tt_tiling tdW,
                            int id_dtype, const void *ids, float scale, const void *const *dX, void *const *dW,
                            void *workspace, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------- policy loss */

/* Token t with logits x_t (a row of the chain's output), z = scale * x_t, p = softmax(z):
 *   logp_t  = z[actions[t]] - log sum exp z
 *   ratio_t = exp(logp_t - old_logp[t])
 *   L_t     = -min(ratio_t A_t, clip(ratio_t, 1 - clip_low, 1 + clip_high) A_t)
 *             + kl * (exp(ref_logp[t] - logp_t) - 1 - (ref_logp[t] - logp_t))
 *   loss    = sum_t weight[t] L_t
 *   dX[t]   = weight[t] * dL_t/dlogp_t * scale * (onehot(actions[t]) - p),   dL/dlogp = 0 through a clipped ratio.
 * A token does not count - log probability 0, no loss, a gradient of zeros, whatever its logits hold - if its weight is 0,
 * its action lies outside [0, vocab), or all its logits are -inf.  Logits of -inf have probability 0.  A NaN or +inf in a
 * row that counts gives NaN, as the formulas do. */
typedef struct {
    float scale;               /* of the logits (1 / temperature): finite, above 0 */
    float clip_low, clip_high; /* not negative */
    float kl;                  /* 0: ref_logp is not read and may be NULL */
} tt_policy;

/* X: tokens x vocab under tX;  dX: the same under tdX, or NULL (no gradient; tdX is ignored);  dtype of both TT_F32 | TT_BF16;
 * statistics and sums fp32, equal calls give equal bits.  actions: id_dtype;  old_logp, ref_logp, advantage, weight, logp
 * (written; may be NULL): fp32, one per token;  loss: one fp32 value (written).
 * Workspace: device memory, 256-byte aligned, at least tt_policy_workspace_bytes (with the same tilings; with_dx = 0 if dX
 * will be NULL: the two differ, and neither covers the other).  What is enough for so many tokens is enough for fewer. */
tt_status tt_policy_workspace_bytes(int64_t tokens, int64_t vocab, int k, int dtype, tt_tiling tX, tt_tiling tdX, int with_dx,
                                    size_t *bytes);
tt_status tt_policy_loss(const tt_policy *policy, int64_t tokens, int64_t vocab, int k, int dtype, tt_tiling tX, tt_tiling tdX,
                         const void *const *X, int id_dtype, const void *actions, const float *old_logp, const float *ref_logp,
                         const float *advantage, const float *weight, float *loss, float *logp, void *const *dX,
                         void *workspace, size_t ws_bytes, void *stream);

/* logp[t] = log softmax(scale * x_t)[ids[t]] alone (what a generating or a reference model's logits are asked for); 0 where
 * ids[t] lies outside [0, vocab) or all logits are -inf.  Workspace as above with with_dx = 0. */
tt_status tt_token_logp(int64_t tokens, int64_t vocab, int k, int dtype, tt_tiling tX, float scale, const void *const *X,
                        int id_dtype, const void *ids, float *logp, void *workspace, size_t ws_bytes, void *stream);

/* ------------------------------------------------ activations kept in 8 bits
 * The 8-bit form of a rows x cols tensor under a tiling: per shard Q (int8, the shard's shape) and S (uint8, one per block
 * of 32 columns of a row, blocks counted from the shard's first column, the last one short: srows x ceil(scols / 32)).
 * A value is Q * 2^(S - 127), for any Q and any S but 255.  2^(S - 127) is, as tt_pack8 makes it, the smallest power of two (not
 * below 2^-126) that keeps the block's values within +-127 steps; Q is the value rounded to the nearest step (ties to even), but one
 * step at least where the value is not 0, so that signs, and with them ReLU's gates, stay as they were.  A block with a NaN or
 * an infinity has S = 255 and stands for NaN throughout.  A power of two and eight bits are exact in bf16 and in fp32: unpacking
 * rounds nothing. */
enum { TT_PACK8_BLOCK = 32 };
tt_status tt_pack8(int64_t rows, int64_t cols, int k, int dtype, tt_tiling t, const void *const *X, int8_t *const *Q,
                   uint8_t *const *S, void *stream);
tt_status tt_unpack8(int64_t rows, int64_t cols, int k, int dtype, tt_tiling t, const int8_t *const *Q, const uint8_t *const *S,
                     void *const *X, void *stream);

/* tt_fc_backward with X and Y in 8 bits: XQ, XS under tX;  YQ, YS under tY (Y ReLU's output; ignored when act is NONE, may then
 * be NULL).  G = dY where Y's value is above 0 (act RELU) or dY;  dX = G W^T;  dW = X^T G.  Results are tt_fc_backward's on the
 * unpacked tensors.  dX may be NULL. */
tt_status tt_fc_packed_workspace_bytes(const tt_layer *layer, int64_t batch, int k, int dtype, tt_tiling tX, tt_tiling tW,
                                       tt_tiling tY, tt_tiling tdY, tt_tiling tdX, const uint8_t *forms_dgrad,
                                       const uint8_t *forms_wgrad, int with_dx, size_t *bytes);
tt_status tt_fc_backward_packed(const tt_layer *layer, int64_t batch, int k, int dtype, tt_tiling tX, tt_tiling tW,
                                tt_tiling tY, tt_tiling tdY, tt_tiling tdX, const uint8_t *forms_dgrad,
                                const uint8_t *forms_wgrad, const int8_t *const *XQ, const uint8_t *const *XS,
                                const void *const *W, const int8_t *const *YQ, const uint8_t *const *YS,
                                const void *const *dY, void *const *dX, void *const *dW, void *workspace, size_t ws_bytes,
                                void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TENSOR_TILING_TOKENS_H */
