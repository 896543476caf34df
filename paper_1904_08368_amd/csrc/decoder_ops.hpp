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
  double* logits;       // [splits][tokens][experts]
  int splits;           // parts of the channels whose sums are left apart
};
constexpr int kRouteExperts = 1024, kRouteTopK = 64, kRouteChannels = 1 << 24;   // (channels: what 32-bit places in a row leave room for)
size_t route_workspace_need(const RouteArgs& a);    // of this call
size_t route_workspace_bytes(const RouteArgs& a);   // of it and of any with fewer tokens
hipError_t launch_route(const RouteArgs& a, int dtype, hipStream_t st);

enum : int { A_SILU = 0, A_GELU = 1 };  // RELAY_ACT_*

struct ExpertsArgs {
  int tokens, top_k, channels, inter, experts, group, zeros, act;
  int64_t x_stride, y_stride;
  const void* x;
  const int32_t* chosen;
  const float* weights;
  const void* gate_up;
  const void* down;
  const void* res;
  void* y;
  void* workspace;
  // set by the launcher, as is: pairs of a token and an expert; whether a launch has a workgroup to a pair (or to an expert)
  int pairs, by_pair;
  FastDiv fd_top_k;
  void* h;        // [pairs][inter]
  float* parts;   // [pairs][channels]
  int* sorted;    // [pairs]
  int* blocks;    // [most_blocks][3]
  int most_blocks;
  // (a group as long as the row is the row's chunks of 128, whole, as for the dense layers)
  __host__ __device__ int group_of(int k) const { return group < k ? group : (k + 127) / 128 * 128; }
};
// of the packed weights that a call reads
inline size_t experts_packed_bytes(const ExpertsArgs& a, bool up) {
  return up ? w4_layout(a.experts * 2 * a.inter, a.channels, a.group_of(a.channels), a.zeros != 0).bytes : w4_layout(a.experts * a.channels, a.inter, a.group_of(a.inter), a.zeros != 0).bytes;
}
size_t experts_workspace_bytes(const ExpertsArgs& a);
hipError_t launch_experts(const ExpertsArgs& a, int dtype, hipStream_t st);

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
  void* workspace;  // NULL: a workgroup to a row
  int scale_bits;   // set by the launcher
};
constexpr int kVocab = 1 << 20;
size_t sample_workspace_need(const SampleArgs& a);    // of this call
size_t sample_workspace_bytes(const SampleArgs& a);   // of it and of any with fewer rows
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t st);

}  // namespace relay
