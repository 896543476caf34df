// C-ABI layer of a decoder's operators beside its attention layer (relay_decoder.h): argument checks on the host, then dispatch.
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "../../include/relay_decoder.h"
#include "api_common.hpp"
#include "decoder_ops.hpp"

namespace {

using relay::aligned;
using relay::device_status;
using relay::fail;

size_t esize(int dtype) { return dtype == RELAY_F32 ? 4 : dtype == RELAY_F16 || dtype == RELAY_BF16 ? 2 : 0; }

// a stride that keeps rows of `what` apart
bool apart(int64_t stride, int rows, int64_t what) { return rows <= 1 ? stride >= 0 : stride >= what; }

// `rows` pieces of `bytes` bytes, `stride` bytes from one to the next
struct Operand {
  const void* at;
  size_t bytes;
  int64_t rows = 1;
  uint64_t stride = 0;
};
// whether any of an operand lies within `size` bytes from `from` on
bool overlap(const Operand& o, const void* from, size_t size) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(o.at), q = reinterpret_cast<uintptr_t>(from);
  if (!o.at || !from || !o.bytes || !size || o.rows <= 0 || p >= q + size) return false;
  if (p + o.bytes > q) return true;
  if (o.stride == 0) return false;
  const uintptr_t i = (q - p - o.bytes) / o.stride + 1;   // the first piece that ends behind q
  return i < (uintptr_t)o.rows && p + i * o.stride < q + size;
}

relay_status check_workspace(const void* workspace, size_t bytes, size_t need, std::initializer_list<Operand> operands) {
  if (!workspace || bytes < need) return fail(RELAY_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? bytes : 0, need);
  if (!aligned(workspace, 256)) return fail(RELAY_ERR_ALIGN, "workspace must be 256-byte aligned");
  for (const Operand& o : operands)
    if (overlap(o, workspace, need)) return fail(RELAY_ERR_UNSUPPORTED, "the workspace must not overlap an operand");
  return RELAY_OK;
}

}  // namespace

extern "C" {

relay_status relay_residual_norm(const relay_residual_norm_desc* d, const void* x, const void* residual, const void* gate,
                                 const float* post_weight, const float* post_bias, const float* pre_weight, const float* pre_bias,
                                 void* sum, void* y, void* hip_stream) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  const size_t es = esize(d->dtype);
  if (!es) return fail(RELAY_ERR_DTYPE, "residual norm takes F16, BF16 or F32");
  if (d->tokens < 0 || d->channels <= 0 || d->channels * es > relay::kNormRowBytes)
    return fail(RELAY_ERR_SHAPE, "bad extent (tokens=%d channels=%d, rows of up to %zu bytes)", d->tokens, d->channels, relay::kNormRowBytes);
  if (d->post < RELAY_NORM_NONE || d->post > RELAY_NORM_LAYER || d->pre < RELAY_NORM_NONE || d->pre > RELAY_NORM_LAYER)
    return fail(RELAY_ERR_UNSUPPORTED, "unknown norm (post=%d pre=%d)", d->post, d->pre);
  // (written so that a NaN is refused)
  if (!(d->post_eps >= 0) || !(d->pre_eps >= 0) || !std::isfinite(d->post_eps) || !std::isfinite(d->pre_eps) || !std::isfinite(d->branch_scale) ||
      !std::isfinite(d->residual_scale))
    return fail(RELAY_ERR_SHAPE, "eps must be at least 0, eps and scales finite");
  if (d->x_stride < 0 || d->residual_stride < 0 || d->gate_stride < 0 || !apart(d->sum_stride, d->tokens, sum ? d->channels : 0) ||
      !apart(d->y_stride, d->tokens, y ? d->channels : 0))
    return fail(RELAY_ERR_SHAPE, "strides must not be negative, those of sum and y not below a row");
  if (d->tokens == 0) return RELAY_OK;
  if (!x) return fail(RELAY_ERR_NULL, "x is required");
  if (!y != (d->pre == RELAY_NORM_NONE)) return fail(RELAY_ERR_NULL, "y must be given exactly if there is a norm of the sum");
  if (!sum && !y) return fail(RELAY_ERR_NULL, "one of sum and y is required");
  if ((d->post == RELAY_NORM_NONE && (post_weight || post_bias)) || (d->pre == RELAY_NORM_NONE && (pre_weight || pre_bias)))
    return fail(RELAY_ERR_UNSUPPORTED, "weights and biases of a norm that is not there");
  if (!aligned(x, es) || !aligned(residual, es) || !aligned(gate, es) || !aligned(sum, es) || !aligned(y, es) || !aligned(post_weight, 4) ||
      !aligned(post_bias, 4) || !aligned(pre_weight, 4) || !aligned(pre_bias, 4))
    return fail(RELAY_ERR_ALIGN, "tensors must be aligned to their type");
  if (sum == y) return fail(RELAY_ERR_UNSUPPORTED, "sum and y must not alias each other");
  // a row is read whole by the threads that write it, so an output may stand where an input does, row on row
  const struct { const void* in; int64_t stride; } inputs[] = {{x, d->x_stride}, {residual, d->residual_stride}, {gate, d->gate_stride}};
  for (const auto& i : inputs)
    if (i.in && d->tokens > 1 && ((i.in == sum && i.stride != d->sum_stride) || (i.in == y && i.stride != d->y_stride)))
      return fail(RELAY_ERR_UNSUPPORTED, "an output in the place of an input needs its stride");
  relay::NormArgs a;
  memset(&a, 0, sizeof(a));
  a.tokens = d->tokens; a.channels = d->channels; a.post = d->post; a.pre = d->pre;
  a.post_eps = d->post_eps; a.pre_eps = d->pre_eps; a.branch_scale = d->branch_scale; a.residual_scale = d->residual_scale;
  a.x = x; a.res = residual; a.gate = gate; a.sum = sum; a.y = y;
  a.post_weight = post_weight; a.post_bias = post_bias; a.pre_weight = pre_weight; a.pre_bias = pre_bias;
  a.x_stride = d->x_stride; a.res_stride = d->residual_stride; a.gate_stride = d->gate_stride; a.sum_stride = d->sum_stride; a.y_stride = d->y_stride;
  return device_status(relay::launch_residual_norm(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "residual norm launch");
}

static relay_status route_args(const relay_route_desc* d, relay::RouteArgs* out) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (d->dtype != RELAY_F16 && d->dtype != RELAY_BF16) return fail(RELAY_ERR_DTYPE, "the router takes F16 or BF16");
  if (d->tokens < 0 || d->channels <= 0 || d->channels > relay::kRouteChannels || d->experts <= 0 || d->experts > relay::kRouteExperts)
    return fail(RELAY_ERR_SHAPE, "bad extent (tokens=%d channels=%d experts=%d, channels in 1 .. %d, experts in 1 .. %d)", d->tokens, d->channels, d->experts, relay::kRouteChannels,
                relay::kRouteExperts);
  if (d->top_k <= 0 || d->top_k > d->experts || d->top_k > relay::kRouteTopK)
    return fail(RELAY_ERR_SHAPE, "top_k=%d must be in 1 .. min(experts, %d)", d->top_k, relay::kRouteTopK);
  if (d->channels % 8) return fail(RELAY_ERR_ALIGN, "channels=%d must be a multiple of 8", d->channels);
  if (d->score != RELAY_SCORE_SOFTMAX && d->score != RELAY_SCORE_SIGMOID) return fail(RELAY_ERR_UNSUPPORTED, "unknown score %d", d->score);
  if (d->normalize != 0 && d->normalize != 1) return fail(RELAY_ERR_UNSUPPORTED, "normalize=%d (0 or 1)", d->normalize);
  if (!std::isfinite(d->scale)) return fail(RELAY_ERR_SHAPE, "scale must be finite");
  if (d->x_stride < 0) return fail(RELAY_ERR_SHAPE, "x_stride must not be negative");
  if (d->x_stride % 8) return fail(RELAY_ERR_ALIGN, "x_stride must be a multiple of 8");
  relay::RouteArgs a;
  memset(&a, 0, sizeof(a));
  a.tokens = d->tokens; a.channels = d->channels; a.experts = d->experts; a.top_k = d->top_k; a.score = d->score; a.normalize = d->normalize;
  a.scale = d->scale; a.x_stride = d->x_stride;
  *out = a;
  return RELAY_OK;
}

relay_status relay_route_workspace_bytes(const relay_route_desc* d, size_t* bytes) {
  if (!bytes) return fail(RELAY_ERR_NULL, "bytes is NULL");
  relay::RouteArgs a;
  if (relay_status st = route_args(d, &a)) return st;
  *bytes = a.tokens ? relay::route_workspace_bytes(a) : 0;
  return RELAY_OK;
}

relay_status relay_route(const relay_route_desc* d, const void* x, const void* w, const float* bias, int32_t* chosen, float* weights,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  relay::RouteArgs a;
  if (relay_status st = route_args(d, &a)) return st;
  if (a.tokens == 0) return RELAY_OK;
  if (!x || !w || !chosen || !weights) return fail(RELAY_ERR_NULL, "x, w, chosen and weights are required");
  if (!aligned(x, 16) || !aligned(w, 16)) return fail(RELAY_ERR_ALIGN, "x and w must be 16-byte aligned");
  if (!aligned(bias, 4) || !aligned(chosen, 4) || !aligned(weights, 4)) return fail(RELAY_ERR_ALIGN, "bias, chosen and weights must be aligned to their type");
  if (static_cast<const void*>(chosen) == weights || chosen == x || weights == x || chosen == w || weights == w || (bias && (weights == bias || static_cast<const void*>(chosen) == bias)))
    return fail(RELAY_ERR_UNSUPPORTED, "an output must not alias another operand");
  const size_t row = (size_t)a.channels * 2, choices = (size_t)a.tokens * a.top_k * 4;
  if (relay_status st = check_workspace(workspace, workspace_bytes, relay::route_workspace_need(a),
                                        {{x, row, a.tokens, (uint64_t)a.x_stride * 2}, {w, (size_t)a.experts * row}, {bias, (size_t)a.experts * 4}, {chosen, choices}, {weights, choices}}))
    return st;
  a.x = x; a.w = w; a.bias = bias; a.chosen = chosen; a.weights = weights; a.workspace = workspace;
  return device_status(relay::launch_route(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "router launch");
}

static relay_status experts_args(const relay_experts_w4_desc* d, relay::ExpertsArgs* out) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (d->dtype != RELAY_F16 && d->dtype != RELAY_BF16) return fail(RELAY_ERR_DTYPE, "4-bit experts take F16 or BF16");
  if (d->tokens < 0 || d->top_k <= 0 || d->top_k > relay::kRouteTopK || d->channels <= 0 || d->inter <= 0 || d->experts <= 0 || d->experts > relay::kRouteExperts)
    return fail(RELAY_ERR_SHAPE, "bad extent (tokens=%d top_k=%d channels=%d inter=%d experts=%d)", d->tokens, d->top_k, d->channels, d->inter, d->experts);
  if (d->channels % 16 || d->inter % 16) return fail(RELAY_ERR_ALIGN, "channels=%d and inter=%d must be multiples of 16", d->channels, d->inter);
  if (2L * d->experts * d->inter > 0x40000000L || (long)d->experts * d->channels > 0x7ffffff0L || d->channels > 0x7fffff00 / 16)
    return fail(RELAY_ERR_SHAPE, "experts=%d channels=%d inter=%d too large", d->experts, d->channels, d->inter);
  if (d->group <= 0 || d->group % 32) return fail(RELAY_ERR_SHAPE, "group=%d must be a positive multiple of 32", d->group);
  if (d->has_zeros != 0 && d->has_zeros != 1) return fail(RELAY_ERR_UNSUPPORTED, "has_zeros=%d (0 or 1)", d->has_zeros);
  if (d->act != RELAY_ACT_SILU && d->act != RELAY_ACT_GELU) return fail(RELAY_ERR_UNSUPPORTED, "unknown activation %d", d->act);
  if (d->flags & ~(uint32_t)RELAY_HAS_RESIDUAL) return fail(RELAY_ERR_UNSUPPORTED, "unknown flag bits 0x%x", d->flags);
  if (d->x_stride < 0 || !apart(d->y_stride, d->tokens, d->channels)) return fail(RELAY_ERR_SHAPE, "x_stride must not be negative, y_stride not below channels");
  if (d->x_stride % 8) return fail(RELAY_ERR_ALIGN, "x_stride must be a multiple of 8");
  relay::ExpertsArgs a;
  memset(&a, 0, sizeof(a));
  a.tokens = d->tokens; a.top_k = d->top_k; a.channels = d->channels; a.inter = d->inter; a.experts = d->experts; a.group = d->group;
  a.zeros = d->has_zeros; a.act = d->act; a.x_stride = d->x_stride; a.y_stride = d->y_stride;
  *out = a;
  return RELAY_OK;
}

relay_status relay_experts_w4_workspace_bytes(const relay_experts_w4_desc* d, size_t* bytes) {
  if (!bytes) return fail(RELAY_ERR_NULL, "bytes is NULL");
  relay::ExpertsArgs a;
  if (relay_status st = experts_args(d, &a)) return st;
  *bytes = a.tokens ? relay::experts_workspace_bytes(a) : 0;
  return RELAY_OK;
}

relay_status relay_experts_w4(const relay_experts_w4_desc* d, const void* x, const int32_t* chosen, const float* weights, const void* gate_up,
                              const void* down, const void* residual, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
  relay::ExpertsArgs a;
  if (relay_status st = experts_args(d, &a)) return st;
  if (a.tokens == 0) return RELAY_OK;
  if (!x || !chosen || !weights || !gate_up || !down || !y) return fail(RELAY_ERR_NULL, "x, chosen, weights, gate_up, down and y are required");
  if (!residual != !(d->flags & RELAY_HAS_RESIDUAL)) return fail(RELAY_ERR_NULL, "residual must be given exactly if its flag is set");
  if (!aligned(x, 16) || !aligned(gate_up, 16) || !aligned(down, 16)) return fail(RELAY_ERR_ALIGN, "x, gate_up and down must be 16-byte aligned");
  if (!aligned(y, 2) || !aligned(residual, 2) || !aligned(chosen, 4) || !aligned(weights, 4))
    return fail(RELAY_ERR_ALIGN, "y, residual, chosen and weights must be aligned to their type");
  if (y == x || y == gate_up || y == down || y == chosen || y == weights || y == workspace) return fail(RELAY_ERR_UNSUPPORTED, "output must not alias an input");
  const size_t row = (size_t)a.channels * 2, choices = (size_t)a.tokens * a.top_k * 4;
  if (relay_status st = check_workspace(workspace, workspace_bytes, relay::experts_workspace_bytes(a),
                                        {{x, row, a.tokens, (uint64_t)a.x_stride * 2}, {chosen, choices}, {weights, choices}, {gate_up, relay::experts_packed_bytes(a, true)},
                                         {down, relay::experts_packed_bytes(a, false)}, {residual, row, a.tokens, (uint64_t)a.y_stride * 2}, {y, row, a.tokens, (uint64_t)a.y_stride * 2}}))
    return st;
  a.x = x; a.chosen = chosen; a.weights = weights; a.gate_up = gate_up; a.down = down; a.res = residual; a.y = y; a.workspace = workspace;
  return device_status(relay::launch_experts(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "experts launch");
}

static relay_status sample_args(const relay_sample_desc* d, relay::SampleArgs* out) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (!esize(d->dtype)) return fail(RELAY_ERR_DTYPE, "logits are F16, BF16 or F32");
  if (d->rows < 0 || d->vocab <= 0 || d->vocab > relay::kVocab)
    return fail(RELAY_ERR_SHAPE, "bad extent (rows=%d vocab=%d, vocab in 1 .. %d)", d->rows, d->vocab, relay::kVocab);
  if (d->logits_stride < 0) return fail(RELAY_ERR_SHAPE, "logits_stride must not be negative");
  relay::SampleArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = d->rows; a.vocab = d->vocab; a.logits_stride = d->logits_stride;
  *out = a;
  return RELAY_OK;
}

relay_status relay_sample_workspace_bytes(const relay_sample_desc* d, size_t* bytes) {
  if (!bytes) return fail(RELAY_ERR_NULL, "bytes is NULL");
  relay::SampleArgs a;
  if (relay_status st = sample_args(d, &a)) return st;
  *bytes = a.rows ? relay::sample_workspace_bytes(a) : 0;
  return RELAY_OK;
}

relay_status relay_sample(const relay_sample_desc* d, const void* logits, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, const float* uniform, int32_t* tokens, float* probs, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
  relay::SampleArgs a;
  if (relay_status st = sample_args(d, &a)) return st;
  if (a.rows == 0) return RELAY_OK;
  if (!logits || !tokens) return fail(RELAY_ERR_NULL, "logits and tokens are required");
  if (!aligned(logits, esize(d->dtype)) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) ||
      !aligned(uniform, 4) || !aligned(tokens, 4) || !aligned(probs, 4))
    return fail(RELAY_ERR_ALIGN, "tensors must be aligned to their type");
  if (static_cast<const void*>(tokens) == probs || static_cast<const void*>(tokens) == logits || probs == logits)
    return fail(RELAY_ERR_UNSUPPORTED, "an output must not alias another operand");
  // (all workgroups of a row read its settings, one writes its outputs)
  const size_t numbers = (size_t)a.rows * 4;
  for (const void* in : {static_cast<const void*>(temperature), static_cast<const void*>(top_k), static_cast<const void*>(top_p), static_cast<const void*>(min_p),
                         static_cast<const void*>(uniform)})
    if (overlap({tokens, numbers}, in, numbers) || overlap({probs, numbers}, in, numbers)) return fail(RELAY_ERR_UNSUPPORTED, "an output must not overlap a setting");
  if (workspace) {
    const size_t need = relay::sample_workspace_need(a);
    const size_t es = esize(d->dtype);
    if (relay_status st = check_workspace(workspace, workspace_bytes, need,
                                          {{logits, a.vocab * es, a.rows, (uint64_t)a.logits_stride * es}, {temperature, numbers}, {top_k, numbers}, {top_p, numbers}, {min_p, numbers},
                                           {uniform, numbers}, {tokens, numbers}, {probs, numbers}}))
      return st;
    a.workspace = need ? workspace : nullptr;
  }
  a.logits = logits; a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.uniform = uniform;
  a.tokens = tokens; a.probs = probs;
  return device_status(relay::launch_sample(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "sampling launch");
}

}  // extern "C"
