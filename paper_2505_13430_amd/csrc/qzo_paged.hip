// Attention of the newest tokens of sequences over a paged cache of keys and values.
#include <algorithm>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {

// One wavefront per row and query head; a lane holds DH/64 features.  out = sum_k exp(s_k - max) v_k / sum_k exp(s_k - max),
// s_k = scale q . k, in one pass with the running maximum and sum.
template <int DH, bool E4M3>
__global__ __launch_bounds__(256) void paged_attention_kernel(PagedArgs a) {
  constexpr int E = DH / 64;
  const uint32_t lane = threadIdx.x & 63u;
  const uint64_t w = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6);
  const uint32_t row = (uint32_t)(w / a.q_heads), h = (uint32_t)(w % a.q_heads), kh = h / a.group;
  uint32_t seq = row, behind = 0;               // tokens of the sequence behind this row's
  if (a.starts) {
    if (row >= a.n_rows || (int32_t)row >= a.starts[a.n_seq]) return;
    uint32_t lo = 0, hi = a.n_seq;
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) >> 1;
      if (a.starts[mid] <= (int32_t)row) lo = mid; else hi = mid;
    }
    seq = lo;
    behind = (uint32_t)a.starts[seq + 1] - 1u - row;
  }
  if (seq >= a.n_seq || row >= a.n_rows) return;
  const int64_t room = (int64_t)a.max_blocks << a.block_shift;
  int64_t len = (int64_t)a.lengths[seq];
  len = min(len, room) - (int64_t)behind;
  float q[E], acc[E], m = -INFINITY, l = 0.0f;
  const float ks = (a.k_scale ? a.k_scale[kh] : 1.0f) * a.scale * 1.44269504f, vs = a.v_scale ? a.v_scale[kh] : 1.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = bf16_to_f32(a.q[(uint64_t)row * a.ld_q + h * DH + lane * E + e]);
    acc[e] = 0.0f;
  }
  for (int64_t k = 0; k < len; ++k) {
    const uint32_t id = (uint32_t)a.tables[(uint64_t)seq * a.max_blocks + (uint32_t)(k >> a.block_shift)];
    if (id >= a.n_blocks) continue;
    const uint64_t at = (((((uint64_t)id * a.kv_heads + kh) << a.block_shift) + ((uint32_t)k & ((1u << a.block_shift) - 1u))) * DH) + lane * E;
    float s = 0.0f, v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float kk;
      if (E4M3) {
        kk = __builtin_amdgcn_cvt_f32_fp8((int)((const unsigned char*)a.k)[at + e], 0);
        v[e] = __builtin_amdgcn_cvt_f32_fp8((int)((const unsigned char*)a.v)[at + e], 0);
      } else {
        kk = bf16_to_f32(((const bf16_t*)a.k)[at + e]);
        v[e] = bf16_to_f32(((const bf16_t*)a.v)[at + e]);
      }
      s = __builtin_fmaf(q[e], kk, s);
    }
    s = wave_sum(s) * ks;
    if (s == -INFINITY) continue;
    const float m2 = fmaxf(m, s), f = exp2f(m - m2), p = exp2f(s - m2);
    l = l * f + p;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(p, v[e], acc[e] * f);
    m = m2;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    a.out[(uint64_t)row * a.ld_out + h * DH + lane * E + e] = (bf16_t)(pack_bf16x2(l == 0.0f ? 0.0f : acc[e] * (vs / l), 0.0f) & 0xffffu);
}

uint64_t paged_attention_scratch(uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }

hipError_t launch_paged_attention(const PagedArgs& a, uint32_t head_dim, bool e4m3, void*, hipStream_t st) {
  const uint32_t rows = a.starts ? a.n_rows : std::min(a.n_rows, a.n_seq);
  const uint32_t wgs = (uint32_t)(((uint64_t)rows * a.q_heads + 3) / 4);
  if (wgs == 0) return hipSuccess;
  if (head_dim == 128) {
    if (e4m3) paged_attention_kernel<128, true><<<wgs, 256, 0, st>>>(a);
    else paged_attention_kernel<128, false><<<wgs, 256, 0, st>>>(a);
  } else {
    if (e4m3) paged_attention_kernel<64, true><<<wgs, 256, 0, st>>>(a);
    else paged_attention_kernel<64, false><<<wgs, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace qzo
