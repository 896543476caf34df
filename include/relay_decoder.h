/*
 * relay_decoder.h -- fused primitive operators of a decoder's step beside its attention layer: the norms of a block with the residual
 * stream, a mixture of experts with 4-bit weights, the choice of the next token.
 *
 * The calling convention of relay_fused.h and relay_attention.h holds here too: static shapes in a descriptor, device pointers that the
 * caller owns, preallocated outputs and scratch, work enqueued on `hip_stream`, argument checks on the host before any HIP call, a status and a
 * message on failure (paper Section 3.3, "Backends").  Strides are in elements, the innermost extent is contiguous.  What a program chooses on
 * the device (experts, settings of a row) is checked there: what names nothing is skipped.  A call without tokens or rows is valid and launches nothing.
 * Workspaces: 256-byte aligned, at least as many bytes as the call's _workspace_bytes says, apart from all operands, zero before their first use, left ready for the next call
 * of the same operator that asks for no more.  What _workspace_bytes says also suffices for fewer tokens or rows of the same descriptor.  Operators, and calls that may run at the same time, need workspaces of their own.
 *
 * One block, beside its attention layer: relay_residual_norm -> relay_route -> relay_experts_w4 -> relay_residual_norm.
 */
#ifndef RELAY_DECODER_H_
#define RELAY_DECODER_H_

#include "relay_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norms of a block, with its gate and the residual stream ---------------------------------------------------- */
enum { RELAY_NORM_NONE = 0, RELAY_NORM_RMS = 1, RELAY_NORM_LAYER = 2 };

typedef struct {
  int32_t dtype;              /* of x, residual, gate, sum and y: RELAY_F16, RELAY_BF16 or RELAY_F32 */
  int32_t tokens, channels;   /* rows of 1 element to 65536 bytes */
  int32_t post, pre;          /* RELAY_NORM_*: of the block's output x; of the sum, for the next block */
  float post_eps, pre_eps;    /* >= 0 */
  float branch_scale, residual_scale;
  int64_t x_stride, residual_stride, gate_stride, sum_stride, y_stride;   /* of rows; gate_stride 0: one gate for all tokens */
} relay_residual_norm_desc;

/* What stands between two blocks, as one primitive function (the elementwise operators and the reductions they feed form one group, paper Section 4.1):
 *   s = residual_scale * residual + branch_scale * gate * post(x),   sum = s,   y = pre(s)
 *   RMS:   v / sqrt(mean(v^2) + eps) * weight + bias        LAYER: (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * weight + bias
 * over the channels of a token, in fp32, each output rounded once; y is made from s before its rounding.
 *   x, residual, gate, sum, y [tokens][channels]; weights and biases fp32 [channels]
 *   residual, gate NULL: not there.  A weight NULL: ones, a bias NULL: zeros; both must be NULL for RELAY_NORM_NONE.
 *   sum NULL: not written.  y must be given exactly if pre is not RELAY_NORM_NONE; one of sum and y must be.
 * sum and y may be x, residual or gate with the same stride (gate only if it has a row for every token); sum and y must not overlap otherwise, nor each other.
 * Any alignment of the element type.  Errors: _NULL, _DTYPE, _SHAPE, _ALIGN, _UNSUPPORTED (kinds, aliasing), _DEVICE. */
relay_status relay_residual_norm(const relay_residual_norm_desc* d, const void* x, const void* residual, const void* gate,
                                 const float* post_weight, const float* post_bias, const float* pre_weight, const float* pre_bias,
                                 void* sum, void* y, void* hip_stream);

/* ---- the router of a mixture of experts ------------------------------------------------------------------------- */
enum { RELAY_SCORE_SOFTMAX = 0, RELAY_SCORE_SIGMOID = 1 };

typedef struct {
  int32_t dtype;              /* of x and w: RELAY_F16 or RELAY_BF16 */
  int32_t tokens, channels;   /* channels a multiple of 8, up to 2^24 */
  int32_t experts, top_k;     /* 1 .. 1024; 1 .. min(experts, 64) */
  int32_t score;              /* RELAY_SCORE_* */
  int32_t normalize;          /* 1: the weights of a token's experts add up to `scale` */
  float scale;
  int64_t x_stride;
} relay_route_desc;

/* The router's product, scores and choice as one primitive function (paper Section 4.1).  chosen[t] = the top_k experts of token t with the largest score + bias, weights[t] = their scores (without bias) [/ their sum] * scale, where
 *   l = w x,   score = softmax(l) over the experts, or 1 / (1 + exp(-l)) each
 * The largest comes first, equal ones in the order of their numbers; a NaN counts as less than everything.  Products, sums and scores are 64-bit, so that a choice does not hang on
 * the order of a sum; weights are rounded once, to fp32.  A sum of zero leaves weights of zero.
 *   x [tokens][channels], 16-byte aligned with x_stride a multiple of 8; w [experts][channels], 16-byte aligned; bias fp32 [experts] or NULL
 *   chosen int32, weights fp32 [tokens][top_k]
 * Errors: _NULL, _DTYPE, _SHAPE, _ALIGN, _UNSUPPORTED (score, normalize, aliasing), _WORKSPACE (the workspace is required), _DEVICE. */
relay_status relay_route_workspace_bytes(const relay_route_desc* d, size_t* bytes);
relay_status relay_route(const relay_route_desc* d, const void* x, const void* w, const float* bias, int32_t* chosen, float* weights,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- the experts ------------------------------------------------------------------------------------------------ */
enum { RELAY_ACT_SILU = 0, RELAY_ACT_GELU = 1 };   /* v / (1 + exp(-v));  v (1 + erf(v / sqrt 2)) / 2 */

typedef struct {
  int32_t dtype;              /* of x, y, the scales and the residual: RELAY_F16 or RELAY_BF16 */
  int32_t tokens, top_k;      /* top_k 1 .. 64 */
  int32_t channels, inter;    /* multiples of 16 */
  int32_t experts;            /* 1 .. 1024 */
  int32_t group, has_zeros;   /* of the 4-bit weights, as of relay_qdense_w4_desc */
  int32_t act;                /* RELAY_ACT_* */
  uint32_t flags;             /* RELAY_HAS_RESIDUAL */
  int64_t x_stride, y_stride; /* of the rows of x; of y and of the residual */
} relay_experts_w4_desc;

/* y[t] = sum_s weights[t][s] * down_e (act(gate_e x[t]) * up_e x[t])  [+ residual[t]],   e = chosen[t][s]
 * for few tokens, where the chosen experts' codes are most of what there is to read: each is read once for 4, 8 or 16 of the tokens that chose it (as many as that are on the
 * mean, from the numbers of tokens and experts), or for 64 where experts have many.
 * act * up is rounded to the tensors' type for the second product (an operand of the matrix cores; past the type's range it is an infinity); sums are fp32, in a fixed order, and
 * weights are applied to them.
 * Two launches for up to 8 or 16 choices, three or four for more (of up to 4096 at a time): what is elementwise goes into the products' ends (paper
 * Section 4.1), scales behind the quantized operands (Section 4.2).
 * gate_up and down are packed by relay_prepack_qdense_w4 with the experts' units one behind the other:
 *   gate_up: n = experts * 2 * inter, k = channels, an expert's gates ahead of its other units;   down: n = experts * channels, k = inter
 * An entry of chosen outside 0 .. experts-1 adds nothing (a padding token has all of them -1 and gets its residual, or zeros); an
 * expert named twice by a token counts twice.
 *   x [tokens][channels], 16-byte aligned with x_stride a multiple of 8; y, residual [tokens][channels] of any alignment of the type; chosen int32,
 *   weights fp32 [tokens][top_k].  y may be the residual; it must not overlap x.
 * Errors: _NULL, _DTYPE, _SHAPE, _ALIGN, _UNSUPPORTED (act, flags, aliasing), _WORKSPACE (the workspace is required), _DEVICE. */
relay_status relay_experts_w4_workspace_bytes(const relay_experts_w4_desc* d, size_t* bytes);
relay_status relay_experts_w4(const relay_experts_w4_desc* d, const void* x, const int32_t* chosen, const float* weights, const void* gate_up,
                              const void* down, const void* residual, void* y, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- the next token --------------------------------------------------------------------------------------------- */
typedef struct {
  int32_t dtype;              /* of the logits: RELAY_F16, RELAY_BF16 or RELAY_F32 */
  int32_t rows, vocab;        /* vocab 1 .. 2^20 */
  int64_t logits_stride;
} relay_sample_desc;

/* One token of each row, in one primitive function from the logits (paper Section 4.1).  With w_i = exp((l_i - max l) / temperature), tokens in descending order of their logits, equal ones in the order of their numbers:
 *   top_k:  the first top_k of them                                       (0 or less: all)
 *   top_p:  of these the shortest run from the first on whose w add up to at least top_p times the sum over them   (1 or more: all)
 *   min_p:  of these the ones with w >= min_p                              (0 or less: all; above 1: none but the first)
 * the first is always kept, and the token is the first kept one at which the running sum of w exceeds uniform times the sum over the kept.
 * temperature 0 (or less): the first.  uniform: in 0 <= u < 1 (less counts as 0, more as the number before 1).  A setting that is NaN is off, a NaN temperature is 1, a NaN uniform 0.
 * A logit that is NaN counts as -infinity; tokens of -infinity are never named.  A row without any other gets token -1 and probability 0; a
 * logit of +infinity shares the row with its like.
 * Weights are evaluated in 64 bits and added up as integers, as multiples of 2^-62 vocab (vocab rounded up to a power of two; 2^-51 where that is more) of the
 * largest, so that a result does not depend on the order of a sum; a weight below half of that is zero.
 *   logits [rows][vocab], any alignment of the type; temperature, top_p, min_p fp32, top_k int32, each [rows] or NULL (1, all, all, all); uniform
 *   fp32 [rows], or NULL: the first of each row
 *   tokens int32 [rows]; probs fp32 [rows] or NULL: w of the token over the sum of w over the kept (1 where the first is what is asked for); neither may overlap a setting
 * Workspace: NULL is valid (few rows then take longer).  Errors: _NULL, _DTYPE, _SHAPE, _ALIGN, _UNSUPPORTED (aliasing), _WORKSPACE, _DEVICE. */
relay_status relay_sample_workspace_bytes(const relay_sample_desc* d, size_t* bytes);
relay_status relay_sample(const relay_sample_desc* d, const void* logits, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, const float* uniform, int32_t* tokens, float* probs, void* workspace, size_t workspace_bytes,
                          void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* RELAY_DECODER_H_ */
