// Internal interface between the C-ABI layer of the attention operators (api_attention.cpp) and their gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fastdiv.hpp"

namespace relay {

enum : int { T_F32 = 0, T_F16 = 1, T_BF16 = 4 };  // relay_dtype

// One tensor of a rotation: heads of `src` go to `dst`.  Strides in elements.
struct RopePart {
  const void* src;
  void* dst;
  int64_t src_token, src_head;
  int64_t dst_token, dst_head;   // dst_token: unused where the token's place comes from the cache
};

struct RopeArgs {
  int parts;                     // 1: a tensor; 3: queries, keys and values of a cache append
  int tokens, heads;             // of all parts together
  int q_heads, qk_heads;         // heads below q_heads: part 0, below qk_heads: part 1, the others: part 2 (not turned)
  int head_dim, rotary_dim, style, inverse, table_rows;
  int num_slots;                 // num_pages * page_size
  FastDiv fd_page;               // by page_size
  int page_size;
  int64_t page_stride, slot_stride;
  const float* cos_sin;
  const int32_t* positions;
  const int32_t* slots;
  RopePart part[3];
  int vec;                       // all tensors can be read and written in 16-byte pieces
  // set by the launcher: pieces of a head that are turned, all of them, groups of heads
  int turn_pieces, pieces, head_groups;
  FastDiv fd_pieces, fd_groups;
};
// false: more threads than one launch holds
bool rope_fits(const RopeArgs& a, int dtype);
hipError_t launch_rope(const RopeArgs& a, int dtype, hipStream_t st);

struct RopeTableArgs {
  int rows, first, pairs, scaling;
  double base, factor, slow, fast, original_len, magnitude;
  float* out;
};
hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t st);

struct AttnArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  const int32_t* page_table;
  const int32_t* q_starts;
  const int32_t* kv_lens;
  int batch, tokens, q_heads, kv_heads, head_dim;
  int group;                     // q_heads / kv_heads
  int num_pages, page_size, pages_per_seq;
  int max_q_len, max_kv_len, causal, window;
  float scale_log2;              // scale * log2(e)
  FastDiv fd_page, fd_group;
  int64_t q_token, out_token, page_stride, slot_stride, head_stride;
  void* workspace;
};
// bytes of the workspace that a call with these extents can use (0: none)
size_t attn_workspace_bytes(const AttnArgs& a);
bool attn_fits(const AttnArgs& a);
hipError_t launch_attention(const AttnArgs& a, int dtype, hipStream_t st);
// the kernel for many rows (paged_attention_tiles.hip)
size_t attn_tiles_workspace_bytes(const AttnArgs& a);
hipError_t launch_attention_tiles(const AttnArgs& a, int dtype, hipStream_t st);

// Packed 4-bit weights.  Units in tiles of 16, the reduction in chunks of 128; a tile's chunk is 64 x 16 bytes, the A operands of four
// 16x16x32 matrix instructions: lane l holds unit l % 16, and its word s the eight codes of i = 32 s + 8 (l / 16) + 0..7, code 2j in
// bits 4j.. and code 2j + 1 in bits 16 + 4j.. of the word before it is turned left (dense_w4.hip).  Behind all codes the scales [tile][group][16] in the
// activations' type, behind them 16 + the zero points [tile][group][16] as bytes.  What lies past n or k is zero.
struct W4Layout {
  int tiles, chunks, groups;
  size_t scales_at, zeros_at, bytes;
};
inline W4Layout w4_layout(int n, int k, int group, bool zeros) {
  W4Layout l;
  l.tiles = (n + 15) / 16;
  l.chunks = (k + 127) / 128;
  l.groups = (k + group - 1) / group;
  l.scales_at = (size_t)l.tiles * l.chunks * 1024;
  l.zeros_at = l.scales_at + (size_t)l.tiles * l.groups * 32;
  l.bytes = l.zeros_at + (zeros ? (size_t)l.tiles * l.groups * 16 : 0);
  return l;
}
struct W4Args {
  const void* x;
  const void* packed;
  const float* bias;
  const void* res;
  void* y;
  int m, n, k, group, zeros, relu;
  int wide;   // four neighbours of y, the residual and the bias can be read and written at once (launch_w4 finds out)
  int64_t x_stride, y_stride;
};
hipError_t launch_w4_pack(const W4Args& a, int dtype, const uint8_t* codes, const void* scales, const uint8_t* zeros, void* packed, hipStream_t st);
bool w4_fits(const W4Args& a);
hipError_t launch_w4(const W4Args& a, int dtype, hipStream_t st);

}  // namespace relay
