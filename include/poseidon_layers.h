/*
 * poseidon_layers.h - layer operators of a pipeline stage on one AMD Instinct
 * MI355X (gfx950): what a stage computes and keeps between the forward node
 * F_{s,m} and the backward node B_{s,m} of a micro-batch.
 *
 * poseidon.h plans a pipeline from tables of layer times and memory.  The
 * operators here are the parts of such layers that those tables depend on:
 * activations kept in 8 bits until the backward pass (they decide how many
 * micro-batches a stage's memory holds), the gated activation and the weight
 * gradients that read what was kept, the sort of tokens by expert with its
 * gather and weighted combination, the experts' products over their rows, the
 * norm with the residual's addition, causal attention over packed sequences,
 * and the embedding of the first stage.
 * Forward and backward are both here.
 *
 * Matrices are row-major in DEVICE memory: `rows` rows of `width` values,
 * neighbouring rows `pitch` values apart (pitch >= width).  Any pitch and any
 * address aligned to the value's own size is accepted.  Sums are held in
 * 32 bits and rounded once, to the output's type, to nearest even.
 *
 * 8-bit form ("stash"): the values of a row in groups of POSEIDON_GROUP share a
 * power-of-two scale 2^e, the least with |x| <= 127 * 2^e for every x of the
 * group, e held to [-126, 121] (POSEIDON_F16: [-24, 9]) so that restored values
 * are finite and exact in the type they came from.  Code = x / 2^e rounded to
 * the nearest whole number, ties to even, held to [-127, 127]; scale byte =
 * e + 127.  A group that holds an infinity or a NaN has scale byte 255 and codes
 * 0, and is restored as NaN.  For `rows` rows of `width` values, with
 * g = ceil(width / POSEIDON_GROUP): int8 codes[rows][g * POSEIDON_GROUP], values past
 * the width 0, and uint8 scales[rows][g], both without gaps; codes on a 16-byte
 * boundary.
 *
 * Errors are poseidon.h's: 0 = OK, negative = error.  All argument checks
 * happen before any HIP call; nothing aborts or throws across this interface.
 * Calls enqueue work on `hip_stream` (a hipStream_t; NULL = the default
 * stream) of the calling thread's current device, which holds the buffers, and
 * never synchronise, allocate or clear memory through the runtime, so they
 * can be captured into a graph.  They keep nothing between calls and may be
 * called from any number of threads.  Workspaces are the caller's: DEVICE
 * memory on a 256-byte boundary, at least as large as the matching
 * *_workspace function says, its contents of no importance before or after.
 * Calls that may run at the same time need workspaces of their own.
 * Outputs may not overlap inputs or each other.  With rows (or tokens) == 0
 * a call writes what depends on no row and returns POSEIDON_OK.
 */
#ifndef POSEIDON_LAYERS_H
#define POSEIDON_LAYERS_H

#include <stdint.h>

#include "poseidon.h"

#ifdef __cplusplus
extern "C" {
#endif

#define POSEIDON_GROUP 64                  /* values that share a scale */
#define POSEIDON_WIDTH_MAX (1u << 20)      /* values in a row */
#define POSEIDON_PITCH_MAX (1u << 24)      /* values from row to row */
#define POSEIDON_ROWS_MAX 0x7fffffffu      /* rows; for experts: tokens * k */
#define POSEIDON_EXPERTS_MAX 511u          /* experts of poseidon_expert_sort and poseidon_expert_product */
#define POSEIDON_RANGES_MAX 65535u         /* row ranges of poseidon_weight_gradient */
#define POSEIDON_TILES_MAX 0x400000u       /* 128 x 128 tiles of all its gradients together */
#define POSEIDON_VOCAB_MAX 0x3ffffffu      /* rows of an embedding table */
#define POSEIDON_NORM_WIDTH_MAX 16384u     /* values in a row of the norm */
#define POSEIDON_HEAD_MAX 128u             /* values of an attention head, a multiple of 8 */
#define POSEIDON_HEADS_MAX 1024u           /* heads of an attention */
#define POSEIDON_SCALE_MAX 0x1p127f        /* of an attention's scores, either sign */

enum { POSEIDON_F32 = 0, POSEIDON_F16 = 1, POSEIDON_BF16 = 2 };   /* value types */

/* ---- activations kept in 8 bits ---- */

/* Keep `rows` rows of x in 8 bits. */
int poseidon_stash(const void *x, uint64_t pitch, uint32_t type, uint64_t rows, uint64_t width, int8_t *codes,
                   uint8_t *scales, void *hip_stream);

/* What was kept, as values of `type` (the one it came from, or any other: then rounded). */
int poseidon_restore(const int8_t *codes, const uint8_t *scales, uint64_t rows, uint64_t width, void *out,
                     uint64_t out_pitch, uint32_t type, void *hip_stream);

/* out = silu(gate) * up, silu(z) = z / (1 + exp(-z)).  With gate_codes, gate_scales, up_codes and up_scales
 * (all or none) gate and up are kept in 8 bits in the same pass. */
int poseidon_gated_forward(const void *gate, uint64_t gate_pitch, const void *up, uint64_t up_pitch, uint32_t type,
                           uint64_t rows, uint64_t width, void *out, uint64_t out_pitch, int8_t *gate_codes,
                           uint8_t *gate_scales, int8_t *up_codes, uint8_t *up_scales, void *hip_stream);

/* Its gradient at the kept gate g and up u: dgate = dout u s (1 + g (1 - s)), dup = dout g s, s = 1 / (1 + exp(-g)). */
int poseidon_gated_backward(const void *dout, uint64_t dout_pitch, uint32_t type, uint64_t rows, uint64_t width,
                            const int8_t *gate_codes, const uint8_t *gate_scales, const int8_t *up_codes,
                            const uint8_t *up_scales, void *dgate, uint64_t dgate_pitch, void *dup, uint64_t dup_pitch,
                            void *hip_stream);

/* Weight gradients of y = x W^T from dy and the kept x: for each range r of rows,
 *   grad[r][o][i] = sum over rows t of the range of dy[t][o] * x[t][i],
 * added to what grad holds where `accumulate` is 1 (the micro-batches of a step).  An empty range gives zeros.
 * offsets: DEVICE int32[n_ranges + 1], non-decreasing, range r = rows [offsets[r], offsets[r + 1]) (each cut to
 *   [0, rows]; empty if it ends before it begins); NULL with n_ranges == 1: all rows.
 * type: of dy, POSEIDON_F16 or POSEIDON_BF16; x is brought to it.  Nothing is lost for POSEIDON_BF16, or if x was kept
 *   from POSEIDON_F16; else what leaves the range of POSEIDON_F16 is held to +-65504, and a value below 2^-14 loses what
 *   lies below 2^-24 (it is rounded toward zero).  grad: [n_ranges][out_width][in_width] of
 *   grad_type without gaps. */
int poseidon_weight_gradient(const void *dy, uint64_t dy_pitch, uint32_t type, uint64_t rows, uint64_t out_width,
                             const int8_t *codes, const uint8_t *scales, uint64_t in_width, const int32_t *offsets,
                             uint32_t n_ranges, void *grad, uint32_t grad_type, uint32_t accumulate, void *workspace,
                             uint64_t workspace_bytes, void *hip_stream);
/* Bytes it needs (0: none, workspace may be NULL); UINT64_MAX if the sizes are refused.  At most 1 GB for 32-bit sums of
 * parts of the rows, and for an out_width that is no multiple of 8 up to 8 GB for a copy of dy. */
uint64_t poseidon_weight_gradient_workspace(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges);

/* ---- tokens by expert ---- */

/* Stable sort of the tokens * k choices (token t's choices at t * k ...) by expert.  A choice outside
 * [0, n_experts) is dropped.
 * order: int32[tokens * k], the choice at each place, the dropped ones at the end;
 * position: int32[tokens * k], the place of each choice, -1 if dropped;
 * offsets: int32[n_experts + 1], expert e's places are [offsets[e], offsets[e + 1]). */
int poseidon_expert_sort(const int32_t *choice, uint64_t tokens, uint32_t k, uint32_t n_experts, int32_t *order,
                         int32_t *position, int32_t *offsets, void *workspace, uint64_t workspace_bytes,
                         void *hip_stream);
uint64_t poseidon_expert_sort_workspace(uint64_t tokens, uint32_t k, uint32_t n_experts);

/* xs[position[t][j]] = x[t]; places past the last choice (from *n_kept, offsets[n_experts] of the sort, to
 * tokens * k) get zeros.  xs: [tokens * k][width] without gaps, or NULL; codes, scales (both or none): the same rows
 * in 8 bits. */
int poseidon_expert_gather(const void *x, uint64_t pitch, uint32_t type, uint64_t tokens, uint64_t width,
                           const int32_t *position, uint32_t k, const int32_t *n_kept, void *xs, int8_t *codes,
                           uint8_t *scales, void *hip_stream);

/* out[t] = sum over j of weights[t][j] * ys[position[t][j]], dropped choices left out, in the order of j; weights:
 * float[tokens][k], or NULL for ones (the gradient of the gather).  ys: [tokens * k][width] without gaps. */
int poseidon_expert_combine(const void *ys, uint32_t type, uint64_t tokens, uint64_t width, const int32_t *position,
                            uint32_t k, const float *weights, void *out, uint64_t out_pitch, void *hip_stream);

/* Its gradient: dys[position[t][j]] = weights[t][j] * dout[t] (places past *n_kept zeros) and
 * dweights[t][j] = <dout[t], ys[position[t][j]]>, 0 for a dropped choice; from the sort's order of all choices. */
int poseidon_expert_combine_backward(const void *dout, uint64_t dout_pitch, const void *ys, uint32_t type,
                                     uint64_t tokens, uint64_t width, const int32_t *order, uint32_t k,
                                     const int32_t *n_kept, const float *weights, void *dys, float *dweights,
                                     void *hip_stream);

/* ---- embedding ---- */

/* out[t] = scale * table[ids[t]]; an id outside [0, vocab) (padding) gives zeros. */
int poseidon_embed(const int32_t *ids, uint64_t tokens, const void *table, uint64_t table_pitch, uint32_t type,
                   uint64_t vocab, uint64_t width, float scale, void *out, uint64_t out_pitch, void *hip_stream);

/* dtable[v] = scale * (sum of dout[t] over the t with ids[t] == v, in a fixed order: the same bits on every call);
 * rows of no token get zeros.  With accumulate == 1 the sums are added and the other rows are not touched. */
int poseidon_embed_backward(const int32_t *ids, uint64_t tokens, const void *dout, uint64_t dout_pitch, uint32_t type,
                            uint64_t vocab, uint64_t width, float scale, void *dtable, uint64_t dtable_pitch,
                            uint32_t dtable_type, uint32_t accumulate, void *workspace, uint64_t workspace_bytes,
                            void *hip_stream);
uint64_t poseidon_embed_backward_workspace(uint64_t tokens, uint64_t vocab, uint64_t width);

/* Rows times the weights of their range: out[t] = W[r] x[t] for the rows t of range r, or with `transposed` 1 W[r]^T x[t],
 * the gradient of the rows.  weights: [n_ranges][out_width][in_width] of `type` without gaps; x has in_width values a row
 * (transposed: out_width), out the other.  type: POSEIDON_F16 or POSEIDON_BF16; out_type: the same, or POSEIDON_F32.
 * offsets: DEVICE int32[n_ranges + 1], non-decreasing, range r = rows [offsets[r], offsets[r + 1]), each cut to
 * [0, rows]; rows before the first and after the last range get zeros.  Offsets that descend leave it open which rows are written.
 * NULL with n_ranges == 1: all rows. */
int poseidon_expert_product(const void *x, uint64_t pitch, uint32_t type, uint64_t rows, const void *weights,
                            uint64_t out_width, uint64_t in_width, uint32_t transposed, const int32_t *offsets,
                            uint32_t n_ranges, void *out, uint64_t out_pitch, uint32_t out_type, void *hip_stream);

/* ---- norm ---- */

/* h = x + residual (residual NULL: x), rstd[t] = 1 / sqrt(mean over the row of h^2 + eps),
 * out[t] = h[t] * rstd[t] * weight; sum[t] = h[t].  sum and rstd may be NULL, and so may out where it is kept in 8 bits.
 * With out_codes and out_scales (both or none) the rows of out are kept in 8 bits, with sum_codes and sum_scales those of
 * h, as they are in `type`.  width <= POSEIDON_NORM_WIDTH_MAX; weight: `width` values of weight_type; eps >= 0. */
int poseidon_norm_forward(const void *x, uint64_t x_pitch, const void *residual, uint64_t residual_pitch, uint32_t type,
                          uint64_t rows, uint64_t width, const void *weight, uint32_t weight_type, float eps, void *out,
                          uint64_t out_pitch, void *sum, uint64_t sum_pitch, float *rstd, int8_t *out_codes,
                          uint8_t *out_scales, int8_t *sum_codes, uint8_t *sum_scales, void *hip_stream);

/* Its gradient at h, from `sum` or from what was kept of it (codes and scales; one of the two): with n = h rstd,
 * g = weight dout: dx = dsum + rstd (g - n mean over the row of n g), which is the gradient of x and of the residual
 * alike, and dweight = sum over the rows of dout n, in a fixed order, added to what dweight holds where `accumulate` is
 * 1.  dsum: the gradient that arrives at `sum`, or NULL.  dweight may be NULL; then it needs no workspace. */
int poseidon_norm_backward(const void *dout, uint64_t dout_pitch, uint32_t type, uint64_t rows, uint64_t width,
                           const void *sum, uint64_t sum_pitch, const int8_t *codes, const uint8_t *scales,
                           const float *rstd, const void *weight, uint32_t weight_type, const void *dsum,
                           uint64_t dsum_pitch, void *dx, uint64_t dx_pitch, float *dweight, uint32_t accumulate,
                           void *workspace, uint64_t workspace_bytes, void *hip_stream);
uint64_t poseidon_norm_backward_workspace(uint64_t rows, uint64_t width);

/* ---- attention ---- */

/* Causal attention of `heads` heads of `dim` values over packed sequences; query head h reads key and value head
 * h / (heads / kv_heads).  For token i of a sequence, over its tokens j up to i:
 *   s[j] = scale <q[i], k[j]>, lse[i] = log sum exp s[j], out[i] = sum of exp(s[j] - lse[i]) v[j].
 * q, k, v, out: token t's head h begins at t * token pitch + h * head pitch; both are multiples of 8 and at least dim, the
 * addresses on a 16-byte boundary.  type: POSEIDON_F16 or POSEIDON_BF16 (exp(s - ...) is rounded to it for the product with v).
 * dim: a multiple of 8 up to POSEIDON_HEAD_MAX; kv_heads divides heads.  lse: float[heads][tokens].
 * offsets: DEVICE int32[sequences + 1], non-decreasing, sequence r = tokens [offsets[r], offsets[r + 1]), each cut to
 * [0, tokens]; tokens before the first and after the last sequence get zeros, their lse -infinity.  Offsets that descend leave
 * it open which tokens are written.  NULL with sequences == 1: all tokens.  POSEIDON_E_RANGE where
 * heads * (tokens / 128 + sequences) passes 2^31 - 256.
 * |scale| <= POSEIDON_SCALE_MAX.  <q, k>, and the gradients' sums for q and k, are summed in 32 bits before scale
 * stretches them: what is below 2^-126 there counts as 0.  Where a stretched score passes 2^127 the row's results are NaN.
 * An infinity or a NaN may reach every result of its own sequence, and none of another. */
int poseidon_attention_forward(const void *q, uint64_t q_token, uint64_t q_head, const void *k, uint64_t k_token,
                               uint64_t k_head, const void *v, uint64_t v_token, uint64_t v_head, uint32_t type,
                               uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dim, float scale,
                               const int32_t *offsets, uint32_t sequences, void *out, uint64_t out_token,
                               uint64_t out_head, float *lse, void *hip_stream);

/* Its gradients from dout and what the forward pass gave: with p[i][j] = exp(s[i][j] - lse[i]) and
 * ds[i][j] = p[i][j] (<dout[i], v[j]> - <dout[i], out[i]>): dq[i] = scale * sum over j of ds[i][j] k[j],
 * dk[j] = scale * sum over i of ds[i][j] q[i], dv[j] = sum over i of p[i][j] dout[i], those two over the query heads that share
 * the key, all in a fixed order.  p and ds are rounded to `type` for these products, in f16 after a power of two that keeps them
 * within its range: gradients that f16 holds are as near for a small dout, or a large one, as for one about 1. */
int poseidon_attention_backward(const void *dout, uint64_t dout_token, uint64_t dout_head, const void *q,
                                uint64_t q_token, uint64_t q_head, const void *k, uint64_t k_token, uint64_t k_head,
                                const void *v, uint64_t v_token, uint64_t v_head, const void *out, uint64_t out_token,
                                uint64_t out_head, const float *lse, uint32_t type, uint64_t tokens, uint32_t heads,
                                uint32_t kv_heads, uint32_t dim, float scale, const int32_t *offsets,
                                uint32_t sequences, void *dq, uint64_t dq_token, uint64_t dq_head, void *dk,
                                uint64_t dk_token, uint64_t dk_head, void *dv, uint64_t dv_token, uint64_t dv_head,
                                void *workspace, uint64_t workspace_bytes, void *hip_stream);
/* Bytes it needs: 8 for each token and head, and up to 1 GB for 32-bit sums of parts of the heads that share a key. */
uint64_t poseidon_attention_backward_workspace(uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dim,
                                               uint32_t sequences);

#ifdef __cplusplus
}
#endif

#endif /* POSEIDON_LAYERS_H */
