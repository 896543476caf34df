// Internal interface between the C-ABI layer of a decoder's operators (api_decoder.cpp) and their gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "attention.hpp"

namespace relay {

enum : int { N_NONE = 0, N_RMS = 1, N_LAYER = 2 };  // RELAY_NORM_*

struct NormArgs {
  int tokens, channels;
  int post, pre;
  float post_eps, pre_eps, branch_scale, residual_scale;
  const void* x;
  const void* res;
  const void* gate;
  const float* post_weight;
  const float* post_bias;
  const float* pre_weight;
  const float* pre_bias;
  void* sum;
  void* y;
  int64_t x_stride, res_stride, gate_stride, sum_stride, y_stride;
};
constexpr size_t kNormRowBytes = 65536;   // what a workgroup's registers hold of a row
hipError_t launch_residual_norm(const NormArgs& a, int dtype, hipStream_t st);

enum : int { S_SOFTMAX = 0, S_SIGMOID = 1 };  // RELAY_SCORE_*

struct RouteArgs {
  int tokens, channels, experts, top_k, score, normalize;
  float scale;
  int64_t x_stride;
  const void* x;
  const void* w;
  const float* bias;
  int32_t* chosen;
  float* weights;
  void* workspace;
  unsigned* counters;   // set by the launcher, as is
  double* logits;       // [tokens][experts]
};
constexpr int kRouteExperts = 1024, kRouteTopK = 64;
size_t route_workspace_bytes(const RouteArgs& a);
hipError_t launch_route(const RouteArgs& a, int dtype, hipStream_t st);

struct SampleArgs {
  int rows, vocab;
  int64_t logits_stride;
  const void* logits;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniform;
  int32_t* tokens;
  float* probs;
  int scale_bits;   // set by the launcher
};
constexpr int kVocab = 1 << 20;
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t st);

}  // namespace relay
