// Attention of new tokens over a paged cache:  o = sum_j softmax_j(scale q.k_j) v_j  over the keys a token sees.
// One wave per token and query head: 64 keys at a time, a key to a lane, the running maximum and sum of the softmax in registers.
#include "attention.hpp"

namespace relay {
namespace {

template <typename T>
__global__ __launch_bounds__(64) void attn_simple_kernel(const AttnArgs a) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  __shared__ float qs[256];
  const int lane = (int)threadIdx.x, h = (int)blockIdx.y, b = (int)blockIdx.z, i = (int)blockIdx.x;
  const int start = a.q_starts[b], nq = a.q_starts[b + 1] - start;
  if (i >= nq || start < 0 || start + i >= a.tokens) return;
  const int D = a.head_dim, hk = h / a.group;
  const T* q = static_cast<const T*>(a.q) + (long)(start + i) * a.q_token + (long)h * D;
  for (int d = lane; d < D; d += 64) qs[d] = (float)q[d];
  __syncthreads();
  const int kv = min(max(a.kv_lens[b], 0), (int)min((long)a.pages_per_seq * a.page_size, (long)a.max_kv_len));
  const int p = a.kv_lens[b] - nq + i;
  const int hi = a.causal ? min(kv, p + 1) : kv;
  const int lo = a.window > 0 ? max(0, p - a.window + 1) : 0;
  float m = -__builtin_inff(), l = 0.f, acc[4] = {0, 0, 0, 0};
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = min(j0 + lane, hi - 1);
    const unsigned pg = fast_div((unsigned)j, a.fd_page);
    const int page = a.page_table[(long)b * a.pages_per_seq + pg];
    const bool ok = j0 + lane < hi && (unsigned)page < (unsigned)a.num_pages;
    const long off = (unsigned)page < (unsigned)a.num_pages ? (long)page * a.page_stride + (long)(j - (int)pg * a.page_size) * a.slot_stride + (long)hk * a.head_stride : 0;
    const T* k = static_cast<const T*>(a.k) + off;
    float s = 0.f;
    for (int d = 0; d < D; d += 8) {
      const vec8 t = *reinterpret_cast<const vec8*>(k + d);
      for (int e = 0; e < 8; ++e) s = fmaf((float)t[e], qs[d + e], s);
    }
    s = ok ? s * a.scale_log2 : -__builtin_inff();
    float mx = s;
    for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
    const float mn = fmaxf(m, mx), base = mn == -__builtin_inff() ? 0.f : mn;
    const float alpha = exp2f(m - base), pr = exp2f(s - base);
    float sum = pr;
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
    l = l * alpha + sum;
    m = mn;
    for (int c = 0; c < 4; ++c) acc[c] *= alpha;
    for (int u = 0; u < min(64, hi - j0); ++u) {
      const float pu = __shfl(pr, u, 64);
      const long ou = __shfl(off, u, 64);
      if (!__shfl((int)ok, u, 64)) continue;
      for (int c = 0; c < 4; ++c)
        if (c * 64 + lane < D) acc[c] = fmaf(pu, (float)static_cast<const T*>(a.v)[ou + c * 64 + lane], acc[c]);
    }
  }
  T* o = static_cast<T*>(a.out) + (long)(start + i) * a.out_token + (long)h * D;
  for (int c = 0; c < 4; ++c)
    if (c * 64 + lane < D) o[c * 64 + lane] = (T)(hi > lo ? acc[c] / l : 0.f);
}

}  // namespace

size_t attn_workspace_bytes(const AttnArgs&) { return 0; }
bool attn_fits(const AttnArgs& a) { return a.q_heads < 65536 && a.batch < 65536; }

hipError_t launch_attention(const AttnArgs& a, int dtype, hipStream_t st) {
  const dim3 grid((unsigned)a.max_q_len, (unsigned)a.q_heads, (unsigned)a.batch);
  if (dtype == T_F16) hipLaunchKernelGGL(attn_simple_kernel<_Float16>, grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL(attn_simple_kernel<__bf16>, grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace relay
