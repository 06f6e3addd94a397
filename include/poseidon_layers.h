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
 * gather and weighted combination, and the embedding of the first stage.
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
#define POSEIDON_EXPERTS_MAX 511u          /* experts of poseidon_expert_sort */
#define POSEIDON_RANGES_MAX 65535u         /* row ranges of poseidon_weight_gradient */
#define POSEIDON_TILES_MAX 0x400000u       /* 128 x 128 tiles of all its gradients together */
#define POSEIDON_VOCAB_MAX 0x3ffffffu      /* rows of an embedding table */

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

#ifdef __cplusplus
}
#endif

#endif /* POSEIDON_LAYERS_H */
