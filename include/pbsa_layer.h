/*
 * pbsa_layer.h -- what a layer of the model runs around its block-sparse attention (pbsa.h), in the same library:
 *
 *   pbsa_norm_rotate_fwd / _bwd      norm of the queries and keys for each head and their position rotation, in one pass
 *   pbsa_rotate                      the rotation alone, and its gradient
 *   pbsa_cross_attention_fwd / _bwd  attention of the chunk's tokens to an encoder's states (a prompt, a recording, an image)
 *
 * Conventions are those of pbsa.h: tensor pointers are DEVICE pointers owned by the caller, descriptions are HOST structs
 * guarded by .size, nothing is allocated or synchronised, arguments are checked on the host before any HIP call, results are
 * deterministic (no floating-point atomics, fixed orders of summation), calls may be captured into a graph.
 *
 * Tensors are [n][heads][tokens][d] with element strides {sequence, head, token} and a contiguous last dimension, of the type
 * that .dtype names; 16-byte aligned, strides multiples of 8.  Inputs may have stride 0 (a tensor that all sequences share);
 * outputs may not overlap themselves or, but for what is said below, an input.  Counts of zero are taken: an empty tensor's
 * pointer is not looked at.  Offsets are 64 bits wide.
 */
#ifndef PBSA_LAYER_H
#define PBSA_LAYER_H

#include "pbsa.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PBSA_BF16 0
#define PBSA_FP16 1
#define PBSA_FP32 2 /* pbsa_rotate and pbsa_norm_rotate only */

#define PBSA_ROTARY_MAX_D     256   /* head dim of the rotation: 16 .. 256, a multiple of 16               */
#define PBSA_ROTARY_MAX_AXES  3
#define PBSA_LAYER_MAX_HEADS  4096
#define PBSA_CROSS_MAX_NK     (1 << 24)

/* ---- norm and rotation ------------------------------------------------------------------------------------------------
 * Pair i (of rot / 2) of token t turns by the angle pos[t][axis of i] * freq[i]; the first pairs[0] pairs belong to axis 0,
 * and so on (one axis: the token's place; three: its frame, row and column).  With half = 0 pair i is elements (2i, 2i + 1),
 * with half = 1 (i, i + rot / 2), of the first rot elements of a head; the others pass.
 *     a' = mscale (a cos - b sin),  b' = mscale (a sin + b cos)
 * Angles are formed and reduced to one turn in two pieces of binary64, so that positions may be as far as 2^52; the rest is
 * binary32, rounded once at the end.
 *   pos    [n][T][n_axes] int64, sequences pos_stride_b elements apart (0: all have the same positions)
 *   freq   [rot / 2] binary64, radians per step, with whatever scaling for long contexts the model asks for
 * The norm of a head's row x, weights w (binary32 [d], or NULL: ones):  x w / sqrt(mean(x^2) + eps), sums in binary32. */
typedef struct pbsa_rotary {
  uint32_t size;            /* sizeof(pbsa_rotary)                                                  */
  int32_t dtype;
  int32_t n, T;             /* sequences, tokens of each                                            */
  int32_t Hq, Hk;           /* heads of the two tensors; Hk = 0: there is one tensor, K is not looked at */
  int32_t d, rot;           /* head dim; rotated elements: a multiple of 16, 0 .. d                 */
  int32_t half;             /* 0: pairs (2i, 2i + 1), 1: pairs (i, i + rot / 2)                     */
  int32_t n_axes, pairs[PBSA_ROTARY_MAX_AXES];
  float mscale, eps;
  int64_t pos_stride_b;
  int64_t q[3], k[3];       /* element strides {sequence, head, token} of the inputs                */
  int64_t qo[3], ko[3];     /* of the outputs (backward: of the gradients that come in)             */
  int64_t dq[3], dk[3];     /* backward: of the gradients that go out                               */
} pbsa_rotary;

/* Qo = R Q, Ko = R K; inverse != 0: the transpose (the angles negated, mscale as it is), which is the gradient.  Qo may be Q
 * itself, with the same strides, and Ko K. */
int pbsa_rotate(const pbsa_rotary* p, const void* Q, const void* K, const int64_t* pos, const double* freq, void* Qo, void* Ko,
                int32_t inverse, void* hip_stream);

/* Qo = R norm(Q; wq), Ko = R norm(K; wk).  Qo may be Q itself, with the same strides, and Ko K.  With Ko the ring slots of a
 * cache (pbsa.h) the keys are appended as they are made. */
int pbsa_norm_rotate_fwd(const pbsa_rotary* p, const void* Q, const void* K, const float* wq, const float* wk, const int64_t* pos,
                         const double* freq, void* Qo, void* Ko, void* hip_stream);

/* From the inputs of the forward call and the gradients dQo, dKo of what it wrote: dQ, dK, and the weights' gradients dwq, dwk
 * (binary32 [d], summed over sequences, tokens and heads; NULL where they are not wanted).  dQ may be dQo (strides alike).
 * ws: pbsa_norm_rotate_workspace_bytes(p) bytes, 256-byte aligned. */
int pbsa_norm_rotate_workspace_bytes(const pbsa_rotary* p, size_t* out);
int pbsa_norm_rotate_bwd(const pbsa_rotary* p, const void* Q, const void* K, const float* wq, const float* wk, const int64_t* pos,
                         const double* freq, const void* dQo, const void* dKo, void* dQ, void* dK, float* dwq, float* dwk, void* ws,
                         size_t ws_bytes, void* hip_stream);

/* ---- cross attention --------------------------------------------------------------------------------------------------
 * O = softmax(scale Q K^T over the attended states) V; head h of the Hq query heads reads head h / (Hq / Hk) of K and V.
 *   k_len  [n] int32 or NULL: sequence b has states 0 .. k_len[b] - 1 (a length outside 0 .. Nk: the nearer of the two)
 *   k_mask [n][Nk] bytes or NULL, sequences mask_stride_b apart (0: one mask for all): states with 0 are not attended
 * States that are not attended are never looked at for a result: they may hold anything, NaN included, and their gradients are
 * written as 0.  A row that attends nothing has O = 0, lse = -inf and no gradient.  Scores and sums are binary32; the
 * probabilities, and in the backward pass the gradients of the scores, are rounded to .dtype for the second products.
 *   lse    [n][Hq][T] fp32: logarithm of each row's sum of exp(score); optional in the forward call */
typedef struct pbsa_cross {
  uint32_t size;            /* sizeof(pbsa_cross)                                                   */
  int32_t dtype;            /* PBSA_BF16 or PBSA_FP16                                               */
  int32_t n, T, Nk;         /* sequences, query tokens and encoder states of each                   */
  int32_t Hq, Hk, d;        /* heads (Hk divides Hq), head dim 64 or 128                            */
  float scale;
  int64_t mask_stride_b;
  int64_t q[3], k[3], v[3], o[3];          /* element strides {sequence, head, token}               */
  int64_t dO[3], dq[3], dk[3], dv[3];      /* backward only                                         */
} pbsa_cross;

/* Rows of all heads from 2^29 on are refused (PBSA_ESHAPE) under a mask if the last state lies 4 GiB or more behind the first.
 * ws: pbsa_cross_workspace_bytes(p) bytes of scratch, 256-byte aligned (0 where the call needs none: then ws may be NULL). */
int pbsa_cross_workspace_bytes(const pbsa_cross* p, size_t* out);
int pbsa_cross_attention_fwd(const pbsa_cross* p, const void* Q, const void* K, const void* V, const int32_t* k_len,
                             const uint8_t* k_mask, void* O, float* lse, void* ws, size_t ws_bytes, void* hip_stream);

/* Gradients of the forward call from its inputs, its O and lse, and dO.  dQ, dK and dV are written in full, in .dtype; dK and
 * dV are the sums over the query heads that share a head.  In fp16 the gradients of the scores are scaled into the type's range by
 * the rows' largest |dO|; with values that pass it even so (a sum of |V| over d of more than 2^17) the call is right and slow. */
int pbsa_cross_bwd_workspace_bytes(const pbsa_cross* p, size_t* out);
int pbsa_cross_attention_bwd(const pbsa_cross* p, const void* Q, const void* K, const void* V, const int32_t* k_len,
                             const uint8_t* k_mask, const void* O, const void* dO, const float* lse, void* dQ, void* dK, void* dV,
                             void* ws, size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PBSA_LAYER_H */
