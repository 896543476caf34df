// C-ABI layer of the operators of a cache-served attention layer (relay_attention.h): argument checks on the host, then dispatch.
#include <cmath>
#include <cstring>

#include "../../include/relay_attention.h"
#include "api_common.hpp"
#include "attention.hpp"

namespace {

using relay::aligned;
using relay::device_status;
using relay::fail;

int esize(int dtype) { return dtype == RELAY_F32 ? 4 : dtype == RELAY_F16 || dtype == RELAY_BF16 ? 2 : 0; }

// Rotation geometry shared by the two calls.
relay_status check_rotation(int dtype, int tokens, int head_dim, int rotary_dim, int style, int table_rows) {
  if (!esize(dtype)) return fail(RELAY_ERR_DTYPE, "rope takes F16, BF16 or F32");
  if (tokens < 0 || head_dim <= 0 || table_rows <= 0)
    return fail(RELAY_ERR_SHAPE, "bad extent (tokens=%d head_dim=%d table_rows=%d)", tokens, head_dim, table_rows);
  if (rotary_dim < 2 || rotary_dim > head_dim || rotary_dim % 2)
    return fail(RELAY_ERR_SHAPE, "rotary_dim=%d must be even and in 2 .. head_dim=%d", rotary_dim, head_dim);
  if (style != RELAY_ROPE_HALF && style != RELAY_ROPE_INTERLEAVED) return fail(RELAY_ERR_UNSUPPORTED, "unknown style %d", style);
  return RELAY_OK;
}

// a stride that keeps `what` apart along an axis of `extent`
bool apart(int64_t stride, int extent, int64_t what) { return extent <= 1 ? stride >= 0 : stride >= what; }

relay::RopeArgs rotation(int tokens, int heads, int head_dim, int rotary_dim, int style, int table_rows, const float* cos_sin,
                         const int32_t* positions) {
  relay::RopeArgs a;
  memset(&a, 0, sizeof(a));
  a.parts = 1;
  a.tokens = tokens;
  a.heads = a.q_heads = a.qk_heads = heads;
  a.head_dim = head_dim;
  a.rotary_dim = rotary_dim;
  a.style = style;
  a.table_rows = table_rows;
  a.cos_sin = cos_sin;
  a.positions = positions;
  return a;
}

// the last two conditions of a 16-byte path: whole pieces in every stride, and a table that is read in pairs of entries
bool vec_strides(int es, std::initializer_list<int64_t> strides) {
  for (int64_t s : strides)
    if (s * es % 16) return false;
  return true;
}

}  // namespace

extern "C" {

relay_status relay_rope_table(const relay_rope_table_desc* d, float* cos_sin, void* hip_stream) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (d->rows < 0 || d->first < 0 || d->rotary_dim < 2 || d->rotary_dim % 2)
    return fail(RELAY_ERR_SHAPE, "bad extent (rows=%d first=%d rotary_dim=%d)", d->rows, d->first, d->rotary_dim);
  if (d->scaling < RELAY_ROPE_PLAIN || d->scaling > RELAY_ROPE_BY_PARTS) return fail(RELAY_ERR_UNSUPPORTED, "unknown scaling %d", d->scaling);
  // (written so that a NaN is refused)
  if (!(d->base > 0) || !std::isfinite(d->base) || !std::isfinite(d->magnitude))
    return fail(RELAY_ERR_SHAPE, "base and magnitude must be finite, base > 0");
  if (d->scaling != RELAY_ROPE_PLAIN && (!(d->factor >= 1) || !std::isfinite(d->factor)))
    return fail(RELAY_ERR_SHAPE, "factor must be at least 1");
  if (d->scaling == RELAY_ROPE_BASE && d->rotary_dim == 2) return fail(RELAY_ERR_SHAPE, "RELAY_ROPE_BASE needs rotary_dim > 2");
  if (d->scaling == RELAY_ROPE_BY_PARTS &&
      (!(d->slow >= 0) || !(d->fast > d->slow) || !std::isfinite(d->fast) || !(d->original_len > 0) || !std::isfinite(d->original_len)))
    return fail(RELAY_ERR_SHAPE, "RELAY_ROPE_BY_PARTS needs 0 <= slow < fast and original_len > 0");
  if (d->rows == 0) return RELAY_OK;
  if (!cos_sin) return fail(RELAY_ERR_NULL, "cos_sin is required");
  if (!aligned(cos_sin, 8)) return fail(RELAY_ERR_ALIGN, "cos_sin must be 8-byte aligned");
  const relay::RopeTableArgs a{d->rows, d->first, d->rotary_dim / 2, d->scaling, d->base, d->factor, d->slow, d->fast, d->original_len,
                               d->magnitude, cos_sin};
  return device_status(relay::launch_rope_table(a, static_cast<hipStream_t>(hip_stream)), "rope table launch");
}

relay_status relay_rope(const relay_rope_desc* d, const void* x, const float* cos_sin, const int32_t* positions, void* y,
                        void* hip_stream) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (relay_status st = check_rotation(d->dtype, d->tokens, d->head_dim, d->rotary_dim, d->style, d->table_rows)) return st;
  if (d->heads <= 0) return fail(RELAY_ERR_SHAPE, "heads=%d", d->heads);
  if (d->inverse != 0 && d->inverse != 1) return fail(RELAY_ERR_UNSUPPORTED, "inverse=%d (0 or 1)", d->inverse);
  if (d->x_token_stride < 0 || d->x_head_stride < 0 || !apart(d->y_token_stride, d->tokens, d->head_dim) ||
      !apart(d->y_head_stride, d->heads, d->head_dim))
    return fail(RELAY_ERR_SHAPE, "strides must not be negative, those of y not below head_dim");
  if (d->tokens == 0) return RELAY_OK;
  if (!x || !cos_sin || !positions || !y) return fail(RELAY_ERR_NULL, "x, cos_sin, positions and y are required");
  const int es = esize(d->dtype);
  if (!aligned(x, es) || !aligned(y, es) || !aligned(cos_sin, 8) || !aligned(positions, 4))
    return fail(RELAY_ERR_ALIGN, "x and y must be aligned to their type, cos_sin to 8 bytes, positions to 4");
  if (x == y && (d->x_token_stride != d->y_token_stride || d->x_head_stride != d->y_head_stride))
    return fail(RELAY_ERR_UNSUPPORTED, "a rotation in place needs the same strides on both sides");
  relay::RopeArgs a = rotation(d->tokens, d->heads, d->head_dim, d->rotary_dim, d->style, d->table_rows, cos_sin, positions);
  a.inverse = d->inverse;
  a.part[0] = {x, y, d->x_token_stride, d->x_head_stride, d->y_token_stride, d->y_head_stride};
  a.vec = aligned(x, 16) && aligned(y, 16) && aligned(cos_sin, 16) &&
          vec_strides(es, {d->x_token_stride, d->x_head_stride, d->y_token_stride, d->y_head_stride});
  if (!relay::rope_fits(a, d->dtype)) return fail(RELAY_ERR_SHAPE, "rope: tokens=%d heads=%d exceed one launch", d->tokens, d->heads);
  return device_status(relay::launch_rope(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "rope launch");
}

relay_status relay_rope_append(const relay_rope_append_desc* d, const void* q, const void* k, const void* v, const float* cos_sin,
                               const int32_t* positions, const int32_t* slots, void* q_out, void* k_cache, void* v_cache,
                               void* hip_stream) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (relay_status st = check_rotation(d->dtype, d->tokens, d->head_dim, d->rotary_dim, d->style, d->table_rows)) return st;
  if (d->q_heads <= 0 || d->kv_heads <= 0 || d->num_pages <= 0 || d->page_size <= 0)
    return fail(RELAY_ERR_SHAPE, "non-positive extent (q_heads=%d kv_heads=%d num_pages=%d page_size=%d)", d->q_heads, d->kv_heads,
                d->num_pages, d->page_size);
  if ((long)d->num_pages * d->page_size > 0x7fffffffL) return fail(RELAY_ERR_SHAPE, "the cache exceeds 2^31-1 slots");
  if ((long)d->q_heads + 2L * d->kv_heads > 0x7fffffffL) return fail(RELAY_ERR_SHAPE, "too many heads");
  const int64_t qrow = (int64_t)d->q_heads * d->head_dim;
  if (d->q_token_stride < 0 || d->k_token_stride < 0 || d->v_token_stride < 0 || !apart(d->q_out_token_stride, d->tokens, qrow) ||
      !apart(d->page_stride, d->num_pages, d->head_dim) || !apart(d->slot_stride, d->page_size, d->head_dim) ||
      !apart(d->head_stride, d->kv_heads, d->head_dim))
    return fail(RELAY_ERR_SHAPE, "strides must not be negative, q_out's not below a row, the cache's not below head_dim");
  if (d->tokens == 0) return RELAY_OK;
  if (!q || !k || !v || !cos_sin || !positions || !slots || !q_out || !k_cache || !v_cache)
    return fail(RELAY_ERR_NULL, "every operand is required");
  const int es = esize(d->dtype);
  if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(q_out, es) || !aligned(k_cache, es) || !aligned(v_cache, es) ||
      !aligned(cos_sin, 8) || !aligned(positions, 4) || !aligned(slots, 4))
    return fail(RELAY_ERR_ALIGN, "tensors must be aligned to their type, cos_sin to 8 bytes, positions and slots to 4");
  if (q == q_out && d->q_token_stride != d->q_out_token_stride)
    return fail(RELAY_ERR_UNSUPPORTED, "a rotation in place needs the same stride on both sides");
  if (k_cache == v_cache || k_cache == k || v_cache == v || k_cache == q_out || v_cache == q_out || q_out == k || q_out == v)
    return fail(RELAY_ERR_UNSUPPORTED, "an output must not alias another operand");
  relay::RopeArgs a = rotation(d->tokens, d->q_heads + 2 * d->kv_heads, d->head_dim, d->rotary_dim, d->style, d->table_rows, cos_sin, positions);
  a.parts = 3;
  a.q_heads = d->q_heads;
  a.qk_heads = d->q_heads + d->kv_heads;
  a.num_slots = d->num_pages * d->page_size;
  a.page_size = d->page_size;
  a.fd_page = relay::make_fastdiv((uint32_t)d->page_size);
  a.page_stride = d->page_stride;
  a.slot_stride = d->slot_stride;
  a.slots = slots;
  a.part[0] = {q, q_out, d->q_token_stride, d->head_dim, d->q_out_token_stride, d->head_dim};
  a.part[1] = {k, k_cache, d->k_token_stride, d->head_dim, 0, d->head_stride};
  a.part[2] = {v, v_cache, d->v_token_stride, d->head_dim, 0, d->head_stride};
  a.vec = aligned(q, 16) && aligned(k, 16) && aligned(v, 16) && aligned(q_out, 16) && aligned(k_cache, 16) && aligned(v_cache, 16) &&
          aligned(cos_sin, 16) && vec_strides(es, {d->q_token_stride, d->k_token_stride, d->v_token_stride, d->q_out_token_stride,
                                                   d->head_dim, d->page_stride, d->slot_stride, d->head_stride});
  if (!relay::rope_fits(a, d->dtype)) return fail(RELAY_ERR_SHAPE, "rope: tokens=%d heads=%d exceed one launch", d->tokens, a.heads);
  return device_status(relay::launch_rope(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "rope append launch");
}

static relay_status attention_args(const relay_paged_attention_desc* d, relay::AttnArgs* out) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (d->dtype != RELAY_F16 && d->dtype != RELAY_BF16) return fail(RELAY_ERR_DTYPE, "paged attention takes F16 or BF16");
  if (d->batch < 0 || d->tokens < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->num_pages <= 0 || d->page_size <= 0 ||
      d->pages_per_seq <= 0 || d->max_kv_len < 0 || d->max_q_len < 0)
    return fail(RELAY_ERR_SHAPE, "bad extent (batch=%d tokens=%d q_heads=%d kv_heads=%d num_pages=%d page_size=%d pages_per_seq=%d max_q_len=%d max_kv_len=%d)",
                d->batch, d->tokens, d->q_heads, d->kv_heads, d->num_pages, d->page_size, d->pages_per_seq, d->max_q_len, d->max_kv_len);
  if (d->q_heads % d->kv_heads) return fail(RELAY_ERR_SHAPE, "q_heads=%d must be a multiple of kv_heads=%d", d->q_heads, d->kv_heads);
  if (d->head_dim < 8 || d->head_dim > 256 || d->head_dim % 8)
    return fail(RELAY_ERR_UNSUPPORTED, "head_dim=%d must be a multiple of 8 in 8 .. 256", d->head_dim);
  if (d->causal != 0 && d->causal != 1) return fail(RELAY_ERR_UNSUPPORTED, "causal=%d (0 or 1)", d->causal);
  if (d->window < 0) return fail(RELAY_ERR_SHAPE, "window=%d", d->window);
  if (!std::isfinite(d->scale)) return fail(RELAY_ERR_SHAPE, "scale must be finite");
  const int64_t row = (int64_t)d->q_heads * d->head_dim;
  if (d->q_token_stride < 0 || !apart(d->out_token_stride, d->tokens, row) || d->page_stride < 0 || d->slot_stride < 0 || d->head_stride < 0)
    return fail(RELAY_ERR_SHAPE, "strides must not be negative, out's not below a row");
  if (!vec_strides(2, {d->q_token_stride, d->out_token_stride, d->page_stride, d->slot_stride, d->head_stride}))
    return fail(RELAY_ERR_ALIGN, "strides must be multiples of 8 elements");
  relay::AttnArgs a;
  memset(&a, 0, sizeof(a));
  a.batch = d->batch; a.tokens = d->tokens; a.q_heads = d->q_heads; a.kv_heads = d->kv_heads; a.head_dim = d->head_dim;
  a.group = d->q_heads / d->kv_heads;
  a.num_pages = d->num_pages; a.page_size = d->page_size; a.pages_per_seq = d->pages_per_seq;
  a.max_q_len = d->max_q_len < d->tokens ? d->max_q_len : d->tokens;
  const long held = (long)d->pages_per_seq * d->page_size;
  a.max_kv_len = (long)d->max_kv_len < held ? d->max_kv_len : (int)held;
  a.causal = d->causal; a.window = d->window;
  a.scale_log2 = (float)((double)d->scale * 1.4426950408889634074);
  a.fd_page = relay::make_fastdiv((uint32_t)d->page_size);
  a.fd_group = relay::make_fastdiv((uint32_t)a.group);
  a.q_token = d->q_token_stride; a.out_token = d->out_token_stride;
  a.page_stride = d->page_stride; a.slot_stride = d->slot_stride; a.head_stride = d->head_stride;
  if (!relay::attn_fits(a)) return fail(RELAY_ERR_SHAPE, "paged attention: batch=%d heads=%d and max_kv_len=%d exceed one launch", d->batch, d->q_heads, d->max_kv_len);
  *out = a;
  return RELAY_OK;
}

relay_status relay_paged_attention_workspace_bytes(const relay_paged_attention_desc* d, size_t* bytes) {
  if (!bytes) return fail(RELAY_ERR_NULL, "bytes is NULL");
  relay::AttnArgs a;
  if (relay_status st = attention_args(d, &a)) return st;
  *bytes = a.tokens && a.batch ? relay::attn_workspace_bytes(a) : 0;
  return RELAY_OK;
}

relay_status relay_paged_attention(const relay_paged_attention_desc* d, const void* q, const void* k_cache, const void* v_cache,
                                   const int32_t* page_table, const int32_t* q_starts, const int32_t* kv_lens, void* out,
                                   void* workspace, size_t workspace_bytes, void* hip_stream) {
  relay::AttnArgs a;
  if (relay_status st = attention_args(d, &a)) return st;
  if (a.tokens == 0 || a.batch == 0 || a.max_q_len == 0) return RELAY_OK;
  if (!q || !k_cache || !v_cache || !page_table || !q_starts || !kv_lens || !out)
    return fail(RELAY_ERR_NULL, "every operand but the workspace is required");
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16))
    return fail(RELAY_ERR_ALIGN, "q, out and the cache must be 16-byte aligned");
  if (!aligned(page_table, 4) || !aligned(q_starts, 4) || !aligned(kv_lens, 4))
    return fail(RELAY_ERR_ALIGN, "page_table, q_starts and kv_lens must be 4-byte aligned");
  if (out == q || out == k_cache || out == v_cache) return fail(RELAY_ERR_UNSUPPORTED, "output must not alias an input");
  if (workspace) {
    if (!aligned(workspace, 256)) return fail(RELAY_ERR_ALIGN, "workspace must be 256-byte aligned");
    const size_t need = relay::attn_workspace_bytes(a);
    if (workspace_bytes < need) return fail(RELAY_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    a.workspace = need ? workspace : nullptr;
  }
  a.q = q; a.k = k_cache; a.v = v_cache; a.out = out;
  a.page_table = page_table; a.q_starts = q_starts; a.kv_lens = kv_lens;
  return device_status(relay::launch_attention(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "paged attention launch");
}

static relay_status w4_args(const relay_qdense_w4_desc* d, relay::W4Args* out) {
  if (!d) return fail(RELAY_ERR_NULL, "descriptor is NULL");
  if (d->dtype != RELAY_F16 && d->dtype != RELAY_BF16) return fail(RELAY_ERR_DTYPE, "4-bit dense takes F16 or BF16");
  if (d->m < 0 || d->n <= 0 || d->k <= 0) return fail(RELAY_ERR_SHAPE, "bad extent (m=%d n=%d k=%d)", d->m, d->n, d->k);
  if (d->k % 8) return fail(RELAY_ERR_ALIGN, "k=%d must be a multiple of 8", d->k);
  if (d->k > 0x7fffff00 || d->n > 0x7ffffff0) return fail(RELAY_ERR_SHAPE, "n=%d k=%d too large", d->n, d->k);
  if (d->group <= 0 || d->group % 32) return fail(RELAY_ERR_SHAPE, "group=%d must be a positive multiple of 32", d->group);
  if (d->has_zeros != 0 && d->has_zeros != 1) return fail(RELAY_ERR_UNSUPPORTED, "has_zeros=%d (0 or 1)", d->has_zeros);
  if (d->flags & ~(uint32_t)(RELAY_HAS_BIAS | RELAY_HAS_RESIDUAL | RELAY_RELU)) return fail(RELAY_ERR_UNSUPPORTED, "unknown flag bits 0x%x", d->flags);
  if (d->x_stride < 0 || !apart(d->y_stride, d->m, d->n)) return fail(RELAY_ERR_SHAPE, "x_stride must not be negative, y_stride not below n");
  if (d->x_stride % 8) return fail(RELAY_ERR_ALIGN, "x_stride must be a multiple of 8");
  relay::W4Args a;
  memset(&a, 0, sizeof(a));
  a.m = d->m; a.n = d->n; a.k = d->k;
  // A group as long as the row is the row's chunks of 128, whole: the kernels then apply its scale once a chunk.  (Cut to steps of 32 it was applied at each: 8192 units by
  // 5000, one scale to a unit, fp16, steps / chunks 9.3 / 7.7 us for one row, 24 / 20 for 40, 202 / 158 for 1500.)
  a.group = d->group < d->k ? d->group : (d->k + 127) / 128 * 128;
  a.zeros = d->has_zeros;
  a.relu = (d->flags & RELAY_RELU) != 0;
  a.x_stride = d->x_stride; a.y_stride = d->y_stride;
  if (!relay::w4_fits(a)) return fail(RELAY_ERR_SHAPE, "4-bit dense: m=%d n=%d exceed one launch", d->m, d->n);
  *out = a;
  return RELAY_OK;
}

relay_status relay_qdense_w4_packed_bytes(const relay_qdense_w4_desc* d, size_t* bytes) {
  if (!bytes) return fail(RELAY_ERR_NULL, "bytes is NULL");
  relay::W4Args a;
  if (relay_status st = w4_args(d, &a)) return st;
  *bytes = relay::w4_layout(a.n, a.k, a.group, a.zeros != 0).bytes;
  return RELAY_OK;
}

relay_status relay_prepack_qdense_w4(const relay_qdense_w4_desc* d, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                                     void* packed, size_t packed_bytes, void* hip_stream) {
  relay::W4Args a;
  if (relay_status st = w4_args(d, &a)) return st;
  if (!codes || !scales || !packed) return fail(RELAY_ERR_NULL, "codes, scales and packed are required");
  if ((zeros != nullptr) != (a.zeros != 0)) return fail(RELAY_ERR_NULL, "zeros must be given exactly if has_zeros is set");
  if (!aligned(scales, 2) || !aligned(packed, 16)) return fail(RELAY_ERR_ALIGN, "scales must be 2-byte aligned, packed 16-byte");
  if (packed == codes || packed == scales || packed == zeros) return fail(RELAY_ERR_UNSUPPORTED, "output must not alias an input");
  const size_t need = relay::w4_layout(a.n, a.k, a.group, a.zeros != 0).bytes;
  if (packed_bytes < need) return fail(RELAY_ERR_WORKSPACE, "packed weights of %zu bytes, %zu needed", packed_bytes, need);
  return device_status(relay::launch_w4_pack(a, d->dtype, codes, scales, zeros, packed, static_cast<hipStream_t>(hip_stream)), "4-bit packing launch");
}

relay_status relay_qdense_w4(const relay_qdense_w4_desc* d, const void* x, const void* packed, const float* bias, const void* residual,
                             void* y, void* hip_stream) {
  relay::W4Args a;
  if (relay_status st = w4_args(d, &a)) return st;
  if (a.m == 0) return RELAY_OK;
  if (!x || !packed || !y) return fail(RELAY_ERR_NULL, "x, packed and y are required");
  if (!bias != !(d->flags & RELAY_HAS_BIAS)) return fail(RELAY_ERR_NULL, "bias must be given exactly if its flag is set");
  if (!residual != !(d->flags & RELAY_HAS_RESIDUAL)) return fail(RELAY_ERR_NULL, "residual must be given exactly if its flag is set");
  if (!aligned(x, 16) || !aligned(packed, 16)) return fail(RELAY_ERR_ALIGN, "x and packed must be 16-byte aligned");
  if (!aligned(y, 2) || !aligned(residual, 2) || !aligned(bias, 4)) return fail(RELAY_ERR_ALIGN, "y, residual and bias must be aligned to their type");
  if (y == x || y == packed) return fail(RELAY_ERR_UNSUPPORTED, "output must not alias an input");
  a.x = x; a.packed = packed; a.bias = bias; a.res = residual; a.y = y;
  return device_status(relay::launch_w4(a, d->dtype, static_cast<hipStream_t>(hip_stream)), "4-bit dense launch");
}

}  // extern "C"
