/*
 * relay_attention.h -- fused primitive operators of an attention layer that is served from a paged cache.
 *
 * The calling convention of relay_fused.h holds here too: static shapes in a descriptor, device pointers that the
 * caller owns, preallocated outputs and scratch, work enqueued on `hip_stream`, argument checks on the host before any
 * HIP call, a status and a message on failure (paper Section 3.3, "Backends").  Each entry point is one launch (paper
 * Section 4.1: a primitive function is one kernel) unless said otherwise.  Added here:
 *   - Strides are in elements, the innermost extent (head_dim, k, n) is contiguous.
 *   - Lengths, positions, slots and page numbers are data on the device.  The host cannot check them, so the kernels do: what they
 *     name outside of the tensors that the descriptor states is neither read nor written.
 *   - A call without tokens (tokens == 0, m == 0) is valid and launches nothing.
 *
 * One layer, four launches: relay_qdense_w4 (queries, keys and values of the new tokens) -> relay_rope_append ->
 * relay_paged_attention -> relay_qdense_w4 with the residual.
 */
#ifndef RELAY_ATTENTION_H_
#define RELAY_ATTENTION_H_

#include "relay_fused.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions ------------------------------------------------------------------------------------------
 * The first rotary_dim channels of a head are rotary_dim/2 pairs; pair i of a token at position p is turned by the angle
 * whose cosine and sine are cos_sin[p][i] = (c, s):
 *   y0 = x0 * c - x1 * s,   y1 = x1 * c + x0 * s       (RELAY_ROPE_HALF: channels i and i + rotary_dim/2;
 *                                                       RELAY_ROPE_INTERLEAVED: channels 2i and 2i + 1)
 * in fp32, rounded once to the tensor's type; the other channels are copied.  inverse: by the negative angle.  A
 * rotation's transpose is its inverse, so with inverse = 1 (and a table of magnitude 1, or the same magnitude) the call maps the
 * gradient of y to the gradient of x. */
enum { RELAY_ROPE_HALF = 0, RELAY_ROPE_INTERLEAVED = 1 };

/* How a table stretches its frequencies f_i = base^(-2i/rotary_dim) for contexts longer than the model was trained on:
 *   RELAY_ROPE_PLAIN     f_i
 *   RELAY_ROPE_LINEAR    f_i / factor (positions interpolated)
 *   RELAY_ROPE_BASE      base * factor^(rotary_dim/(rotary_dim-2)) in the place of base; rotary_dim > 2
 *   RELAY_ROPE_BY_PARTS  the interpolation by wavelength of Peng et al. 2023 ("YaRN"): with r = original_len * f_i / (2 pi) turns over
 *                        the original context and g = clamp((r - slow) / (fast - slow), 0, 1):  (1 - g) * f_i / factor + g * f_i */
enum { RELAY_ROPE_PLAIN = 0, RELAY_ROPE_LINEAR = 1, RELAY_ROPE_BASE = 2, RELAY_ROPE_BY_PARTS = 3 };

typedef struct {
  int32_t rows, first;        /* positions first .. first + rows - 1, first >= 0 */
  int32_t rotary_dim;         /* even, >= 2 */
  int32_t scaling;            /* RELAY_ROPE_PLAIN .. */
  double base;                /* > 0 */
  double factor;              /* >= 1 (unused by RELAY_ROPE_PLAIN) */
  double slow, fast;          /* RELAY_ROPE_BY_PARTS: 0 <= slow < fast */
  double original_len;        /* RELAY_ROPE_BY_PARTS: > 0 */
  double magnitude;           /* both entries are multiplied by it; 1 for a rotation */
} relay_rope_table_desc;

/* cos_sin[r][i] = magnitude * (cos, sin)((first + r) * f_i): fp32 [rows][rotary_dim/2][2], device, 8-byte aligned.  Angles are formed and
 * reduced in 64 bits (a position of a million times a 32-bit frequency is off by up to a tenth of a radian).  Made once, kept: what
 * depends on constants alone is evaluated ahead of the run (paper Section 3.3, constant folding). */
relay_status relay_rope_table(const relay_rope_table_desc* d, float* cos_sin, void* hip_stream);

typedef struct {
  int32_t dtype;              /* RELAY_F16, RELAY_BF16 or RELAY_F32 */
  int32_t tokens, heads, head_dim;
  int32_t rotary_dim;         /* even, 2 .. head_dim */
  int32_t style;              /* RELAY_ROPE_HALF or RELAY_ROPE_INTERLEAVED */
  int32_t inverse;            /* 0 or 1 */
  int32_t table_rows;
  int64_t x_token_stride, x_head_stride, y_token_stride, y_head_stride;
} relay_rope_desc;

/* The rotation of a tensor as one primitive function (paper Section 4.1).
 * x, y [tokens][heads][head_dim] with the strides given; cos_sin fp32 [table_rows][rotary_dim/2][2], 8-byte aligned; positions int32 [tokens]:
 * rows of the table.  y may be x (same strides), otherwise they must not overlap.  A token whose position is not a row of the table
 * gets NaN in the channels that are turned.  Any alignment of the element type; 16-byte aligned tensors whose strides are multiples of 16 bytes run faster.
 * Errors: _NULL, _DTYPE, _SHAPE, _UNSUPPORTED (style, inverse), _ALIGN, _DEVICE. */
relay_status relay_rope(const relay_rope_desc* d, const void* x, const float* cos_sin, const int32_t* positions, void* y,
                        void* hip_stream);

typedef struct {
  int32_t dtype;              /* of q, k, v, q_out and the cache: RELAY_F16, RELAY_BF16 or RELAY_F32 */
  int32_t tokens, q_heads, kv_heads, head_dim;
  int32_t rotary_dim, style, table_rows;
  int32_t num_pages, page_size;
  int64_t q_token_stride, k_token_stride, v_token_stride, q_out_token_stride;   /* heads of a token are contiguous */
  int64_t page_stride, slot_stride, head_stride;                                /* of k_cache and of v_cache */
} relay_rope_append_desc;

/* What a decoder does with the projected queries, keys and values of its new tokens, in one launch (the elementwise operators behind a
 * contraction form one group, paper Section 4.1): q_out = rotated q; the rotated
 * keys and the values are stored into the paged cache.
 *   q [tokens][q_heads][head_dim], k, v [tokens][kv_heads][head_dim]: ranges of one projection's rows, or tensors of their own
 *   k_cache, v_cache: element (page, slot, head, channel) at page*page_stride + slot*slot_stride + head*head_stride + channel
 *   slots int32 [tokens]: page * page_size + slot of each token.  A negative one, or one outside the num_pages pages, stores
 *   nothing (a padding token).  Two tokens must not name one slot.
 * q_out may be q (same stride).  A position outside the table makes NaN in the turned channels.  Errors as relay_rope. */
relay_status relay_rope_append(const relay_rope_append_desc* d, const void* q, const void* k, const void* v, const float* cos_sin,
                               const int32_t* positions, const int32_t* slots, void* q_out, void* k_cache, void* v_cache,
                               void* hip_stream);

/* ---- attention of new tokens over a paged cache ---------------------------------------------------------------- */
typedef struct {
  int32_t dtype;              /* of q, out and the cache: RELAY_F16 or RELAY_BF16 */
  int32_t batch;              /* sequences */
  int32_t tokens;             /* rows of q and of out */
  int32_t q_heads, kv_heads;  /* query head h reads key head h / (q_heads / kv_heads) */
  int32_t head_dim;           /* a multiple of 8, 8 .. 256 */
  int32_t num_pages, page_size, pages_per_seq;
  int32_t max_q_len;          /* no sequence has more new tokens, */
  int32_t max_kv_len;         /* ... nor more keys, than this: the launch is sized by them, tokens beyond are not computed, keys beyond not seen */
  int32_t causal;             /* 1: a token sees no key behind its own position */
  int32_t window;             /* > 0: only the last `window` keys up to its own position; 0: all */
  float scale;
  int64_t q_token_stride, out_token_stride;         /* heads of a token are contiguous */
  int64_t page_stride, slot_stride, head_stride;    /* of k_cache and of v_cache */
} relay_paged_attention_desc;

/* The products, the softmax between them and the look-up of the pages as one launch (paper Section 4.1; intermediate results stay off memory),
 * with a second one behind it where more than 16 rows of a key head have their keys shared out.
 * Sequence b has the rows q_starts[b] .. q_starts[b+1]-1 of q (nq of them) as its newest tokens and kv_lens[b] keys in the cache, the new
 * tokens' own among them (relay_rope_append has stored them).  Its token i stands at position p = kv_lens[b] - nq + i and
 *   out = sum_j softmax_j(scale * q . k_j) v_j   over keys 0 <= j < kv_lens[b], j <= p if causal, j > p - window if window > 0
 * Key j lies in slot j % page_size of page page_table[b][j / page_size].  A token that sees no key gets zeros (and so does one whose scores
 * are all -infinity).  Keys that a token does not see do not reach its result, whatever they hold (infinities and NaN included).  Scores, the softmax and the sums
 * are fp32; the probabilities are rounded to the tensor's type for the product with v, whose sums are fp32 (and, where there are more than 16 rows to a key
 * head, for their own sum too).
 * A page number outside 0 .. num_pages-1, or a key past pages_per_seq pages, is not read: such keys count as unseen.
 *   q, out [tokens][q_heads][head_dim] with the token strides given; k_cache, v_cache, strides as relay_rope_append
 *   page_table int32 [batch][pages_per_seq]; q_starts int32 [batch+1], ascending; kv_lens int32 [batch]
 * All tensors 16-byte aligned, strides multiples of 16 bytes.  out must not overlap an input.
 * Where there are few rows and many keys, a sequence's keys are shared out over workgroups that leave partial sums in the
 * workspace; they are joined in a fixed order, so results do not depend on timing.  Workspace contract as of
 * relay_workspace_bytes: 256-byte aligned, at least relay_paged_attention_workspace_bytes(d), zero before its first use, left ready
 * for the next call of any descriptor that asks for no more; NULL is valid (no sharing out, slower). */
relay_status relay_paged_attention_workspace_bytes(const relay_paged_attention_desc* d, size_t* bytes);
relay_status relay_paged_attention(const relay_paged_attention_desc* d, const void* q, const void* k_cache, const void* v_cache,
                                   const int32_t* page_table, const int32_t* q_starts, const int32_t* kv_lens, void* out,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- dense with 4-bit weights ---------------------------------------------------------------------------------- */
typedef struct {
  int32_t dtype;              /* of x, y, the scales and the residual: RELAY_F16 or RELAY_BF16 */
  int32_t m, n, k;            /* k a multiple of 8 */
  int32_t group;              /* weights of a row that share a scale: a multiple of 32; the last group may be short */
  int32_t has_zeros;          /* 0: the zero point of every group is 8 */
  uint32_t flags;             /* RELAY_HAS_BIAS | RELAY_HAS_RESIDUAL | RELAY_RELU */
  int64_t x_stride, y_stride; /* of the rows of x; of y and of the residual */
} relay_qdense_w4_desc;

/* y[m,j] = sum_i x[m,i] * scale[j,i/group] * (code[j,i] - zero[j,i/group])  [+ bias[j]]  [+ residual[m,j]]  [relu]  -> dtype
 * (paper Section 4.2: quantized operands, the scaling fused behind the contraction).  The codes (0..15) and zero points enter the matrix cores as integers; scales are applied to the fp32 sums of a group.
 * relay_prepack_qdense_w4 lays codes, scales and zero points out for the kernels, once (compile-time work): codes uint8 [n][k/2], the
 * even i of a pair in the low four bits; scales [n][ceil(k/group)] of the descriptor's type; zeros uint8 [n][ceil(k/group)], 0..15, NULL
 * exactly if has_zeros is 0.  packed: device, 16-byte aligned, relay_qdense_w4_packed_bytes(d) bytes; it depends on n, k, group,
 * dtype and has_zeros, not on m.
 * x [m][k], 16-byte aligned with x_stride a multiple of 8; y, residual [m][n] of any alignment of the type; bias fp32 [n].
 * y may be the residual; it must not overlap x.  Errors: _NULL, _DTYPE, _SHAPE, _ALIGN, _UNSUPPORTED (flags, aliasing), _WORKSPACE (packed
 * too small), _DEVICE. */
relay_status relay_qdense_w4_packed_bytes(const relay_qdense_w4_desc* d, size_t* bytes);
relay_status relay_prepack_qdense_w4(const relay_qdense_w4_desc* d, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                                     void* packed, size_t packed_bytes, void* hip_stream);
relay_status relay_qdense_w4(const relay_qdense_w4_desc* d, const void* x, const void* packed, const float* bias,
                             const void* residual, void* y, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* RELAY_ATTENTION_H_ */
