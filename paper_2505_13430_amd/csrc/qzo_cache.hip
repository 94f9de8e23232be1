// The paged cache of keys and values: which blocks and slots the newest tokens get (cache_plan_kernel, cache_slots_kernel),
// and the kernel that norms and rotates the heads of q and k and writes k and v to those slots (qk_norm_rope_kernel).
#include <algorithm>
#include <cmath>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {

// ------------------------------------------------------------ block tables and slots ----
// Last i in [0, n) with prefix[i] <= x; prefix ascends, prefix[0] <= x.  Entries that are equal belong to sequences that
// count nothing, the last of them is the one that does.
__device__ __forceinline__ uint32_t last_not_above(const int32_t* prefix, uint32_t n, int32_t x) {
  uint32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (prefix[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// One workgroup.  What sequence i gives back (ended), takes and adds is summed over the sequences before it; the three
// prefixes stay in the LDS, where the blocks and the tokens find their sequence by bisection, so that long prompts are
// spread over all threads.  Every input is read before the first output is written (lengths may be cached, after may be
// before), and no output of this launch is read back: a taken block is found in the free list or in the row of the
// sequence that gives it back, neither of which changes below the stack's old height.
// with_slots: slots and positions too (few tokens); else cache_slots_kernel follows.
constexpr uint32_t PLAN_THREADS = 1024;
__global__ __launch_bounds__(PLAN_THREADS) void cache_plan_kernel(CachePlanArgs a, uint32_t with_slots) {
  extern __shared__ int32_t prefix[];
  int32_t* const back = prefix;                    // [n_seq] blocks given back before sequence i
  int32_t* const take = prefix + a.n_seq;          // [n_seq] blocks taken before it
  int32_t* const start = prefix + 2 * a.n_seq;     // [n_seq] tokens added before it
  int32_t* const old_len = prefix + 3 * a.n_seq;   // [n_seq]
  __shared__ int64_t wave_sums[PLAN_THREADS / 64][3];
  __shared__ int32_t bad;
  const uint32_t tid = threadIdx.x, shift = a.block_shift;
  const int32_t mask = (1 << shift) - 1;
  const int32_t n_free = a.before->n_free;
  const int64_t room = (int64_t)a.max_blocks << shift;
  if (tid == 0) bad = 0;
  __syncthreads();
  const uint32_t per = (a.n_seq + PLAN_THREADS - 1) / PLAN_THREADS, first = tid * per, last = min(first + per, a.n_seq);
  int64_t sum[3] = {0, 0, 0};
  bool wrong = n_free < 0 || (uint32_t)n_free > a.n_blocks, narrow = false;
  for (uint32_t i = first; i < last; ++i) {
    const int32_t have = a.cached[i], add = a.added[i];
    wrong = wrong || have < 0;
    narrow = narrow || have > room || (add > 0 && (int64_t)have + add > room);
    const int64_t held = ((int64_t)have + mask) >> shift;
    sum[0] += add < 0 ? held : 0;
    sum[1] += add < 0 ? 0 : (((int64_t)have + add + mask) >> shift) - held;
    sum[2] += add < 0 ? 0 : add;
    old_len[i] = have;
  }
  if (wrong) atomicOr(&bad, 1);
  if (narrow) atomicOr(&bad, 2);
  // exclusive sums over the threads: within a wavefront, then over the wavefronts before it
  int64_t run[3], total[3];
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    int64_t v = sum[j];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t u = __shfl_up(v, o, 64);
      if ((tid & 63u) >= (uint32_t)o) v += u;
    }
    if ((tid & 63u) == 63u) wave_sums[tid >> 6][j] = v;
    run[j] = v - sum[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    total[j] = 0;
    for (uint32_t w = 0; w < PLAN_THREADS / 64; ++w) {
      if (w == (tid >> 6)) run[j] += total[j];
      total[j] += wave_sums[w][j];
    }
  }
  int32_t status = QZO_OK;
  if (bad & 1) status = QZO_ERR_ARG;
  else if ((bad & 2) || total[2] > (int64_t)a.max_tokens) status = QZO_ERR_SHAPE;
  else if (n_free + total[0] > (int64_t)a.n_blocks) status = QZO_ERR_ARG;        // more blocks than there are
  else if (total[1] > n_free + total[0]) status = QZO_ERR_WORKSPACE;
  const bool ok = status == QZO_OK;
  for (uint32_t i = first; i < last; ++i) {
    const int32_t have = old_len[i], add = a.added[i];
    back[i] = (int32_t)run[0]; take[i] = (int32_t)run[1]; start[i] = (int32_t)run[2];
    const int32_t held = (int32_t)(((int64_t)have + mask) >> shift);
    if (add < 0) run[0] += held;
    else { run[1] += (int32_t)(((int64_t)have + add + mask) >> shift) - held; run[2] += add; }
  }
  __syncthreads();
  for (uint32_t i = first; i < last; ++i) {      // a thread's own sequences: read above, written here
    const int32_t add = a.added[i];
    a.lengths[i] = !ok ? old_len[i] : add < 0 ? 0 : old_len[i] + add;
    a.starts[i] = ok ? start[i] : 0;
  }
  const int32_t n_back = (int32_t)total[0], n_take = ok ? (int32_t)total[1] : 0, n_tok = ok ? (int32_t)total[2] : 0;
  if (tid == 0) {
    a.starts[a.n_seq] = n_tok;
    *a.after = qzo_cache_state{ok ? n_free + n_back - n_take : n_free, n_tok, status, n_take};
  }
  auto given = [&](int32_t r) {                  // r-th block given back
    const uint32_t s = last_not_above(back, a.n_seq, r);
    return a.tables[(uint64_t)s * a.max_blocks + (uint32_t)(r - back[s])];
  };
  auto taken = [&](int32_t k) {                  // k-th block taken: those given back lie on top of the free ones
    return k < n_back ? given(n_back - 1 - k) : a.free[n_free - 1 - (k - n_back)];
  };
  if (ok) {
    for (int32_t k = (int32_t)tid; k < n_take; k += PLAN_THREADS) {
      const uint32_t s = last_not_above(take, a.n_seq, k);
      const uint32_t j = (uint32_t)((old_len[s] + mask) >> shift) + (uint32_t)(k - take[s]);
      a.tables[(uint64_t)s * a.max_blocks + j] = taken(k);
    }
    for (int32_t r = (int32_t)tid; r < n_back - n_take; r += PLAN_THREADS) a.free[n_free + r] = given(r);
  }
  if (!with_slots) return;
  for (uint32_t t = tid; t < a.max_tokens; t += PLAN_THREADS) {
    int32_t slot = -1, at = 0;
    if ((int32_t)t < n_tok) {
      const uint32_t s = last_not_above(start, a.n_seq, (int32_t)t);
      at = old_len[s] + (int32_t)t - start[s];
      const int32_t j = at >> shift, held = (old_len[s] + mask) >> shift;
      const int32_t id = j < held ? a.tables[(uint64_t)s * a.max_blocks + (uint32_t)j] : taken(take[s] + j - held);
      slot = (id << shift) + (at & mask);
    }
    a.slots[t] = slot;
    a.positions[t] = at;
  }
}

// Slots and positions of many tokens, from what cache_plan_kernel left.
__global__ __launch_bounds__(256) void cache_slots_kernel(CachePlanArgs a) {
  extern __shared__ int32_t prefix[];
  for (uint32_t i = threadIdx.x; i <= a.n_seq; i += 256) prefix[i] = a.starts[i];
  __syncthreads();
  const int32_t n_tok = prefix[a.n_seq], mask = (1 << a.block_shift) - 1;
  for (uint32_t t = blockIdx.x * 256u + threadIdx.x; t < a.max_tokens; t += gridDim.x * 256u) {
    int32_t slot = -1, at = 0;
    if ((int32_t)t < n_tok) {
      const uint32_t s = last_not_above(prefix, a.n_seq, (int32_t)t);
      at = a.lengths[s] - (prefix[s + 1] - (int32_t)t);
      slot = (a.tables[(uint64_t)s * a.max_blocks + (uint32_t)(at >> a.block_shift)] << a.block_shift) + (at & mask);
    }
    a.slots[t] = slot;
    a.positions[t] = at;
  }
}

constexpr uint32_t PLAN_SLOTS = 4096;      // tokens whose slots the one workgroup writes itself
hipError_t launch_cache_plan(const CachePlanArgs& a, hipStream_t st) {
  const bool few = a.max_tokens <= PLAN_SLOTS;
  const uint32_t lds = a.n_seq * 16u;
  if (lds > 60u * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)cache_plan_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(CACHE_MAX_SEQ * 16u));
    if (e != hipSuccess) return e;
  }
  cache_plan_kernel<<<1, PLAN_THREADS, lds, st>>>(a, few);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || few) return e;
  cache_slots_kernel<<<std::min<uint32_t>((a.max_tokens + 1023) / 1024, 1024u), 256, (a.n_seq + 1) * 4u, st>>>(a);
  return hipGetLastError();
}

// ------------------------------------------------------------ heads of q and k ----
// y = R(position) (x / sqrt(mean x^2 + eps) * gain), head by head: RMSNorm over the head's DH features, then the pairs
// (i, i + DH/2) turned by position * theta^(-2i/DH).  Everything between the load and the one rounding at the store is
// fp32; the angle is formed in double as a number of turns (position times theta^(-2i/DH) / 2 pi) and only its fraction
// goes to fp32, so that far positions lose nothing.
// DH/8 lanes hold a head, eight features each; a wavefront takes 64 / (DH/8) heads at a time and walks over its share of
// the token's heads with the same angles.
__device__ __forceinline__ float lanes_of_head_sum(float v, int dh) {
  const int n = dh / 8;
  for (int o = 1; o < n; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <int DH>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a, RopeTurns turns, uint32_t parts) {
  constexpr uint32_t LANES = DH / 8, HEADS = 64 / LANES;
  const uint32_t lane = threadIdx.x & 63u, sub = lane % LANES;
  const uint32_t w = blockIdx.x * 4u + (threadIdx.x >> 6), t = w / parts, part = w % parts;
  if (t >= a.n_tokens) return;
  int32_t slot = 0;
  if (a.slots) {
    slot = a.slots[t];
    if (slot < 0 || (uint32_t)slot >= a.n_slots) return;
  }
  const int32_t at = a.positions ? a.positions[t] : (int32_t)((t % a.pass_stride) % a.seq);
  float c[8], s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    c[j] = 1.0f; s[j] = 0.0f;
    if (a.rope) {
      const double turn = (double)at * turns.t[(sub * 8 + j) % (DH / 2)];
      sincospif(2.0f * (float)(turn - rint(turn)), &s[j], &c[j]);
      if (sub < LANES / 2) s[j] = -s[j];
    }
  }
  const uint32_t heads = a.q_heads + a.kv_heads + (a.cache_type ? a.kv_heads : 0u);
  for (uint32_t h = part * HEADS + lane / LANES; h < heads; h += parts * HEADS) {
    const uint4 raw = *reinterpret_cast<const uint4*>(a.qkv + (uint64_t)t * a.ld_qkv + h * DH + sub * 8);
    const uint32_t r[4] = {raw.x, raw.y, raw.z, raw.w};
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(r[j] << 16);
      x[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
    const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.kv_heads;
    const bf16_t* gain = is_q ? a.q_gain : a.k_gain;
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = __builtin_fmaf(x[j], x[j], ss);
    ss = lanes_of_head_sum(ss, DH);
    if (!is_v && gain) {
      const float inv = 1.0f / sqrtf(ss * (1.0f / DH) + a.eps);
      const uint4 g4 = *reinterpret_cast<const uint4*>(gain + sub * 8);
      const uint32_t g[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] *= inv * __uint_as_float(g[j] << 16);
        x[2 * j + 1] *= inv * __uint_as_float(g[j] & 0xffff0000u);
      }
    }
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float other = __shfl_xor(x[j], LANES / 2, 64);
      y[j] = is_v ? x[j] : __builtin_fmaf(other, s[j], x[j] * c[j]);
    }
    if (is_q || !a.cache_type) {
      *reinterpret_cast<uint4*>(a.out + (uint64_t)t * a.ld_out + h * DH + sub * 8) =
          make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
      continue;
    }
    const uint32_t kh = h - a.q_heads - (is_v ? a.kv_heads : 0u);
    const uint64_t row = (((uint64_t)((uint32_t)slot >> a.block_shift) * a.kv_heads + kh) << a.block_shift) + ((uint32_t)slot & ((1u << a.block_shift) - 1u));
    unsigned char* pool = (unsigned char*)(is_v ? a.v : a.k);
    if (a.cache_type == 1) {
      *reinterpret_cast<uint4*>(pool + row * (DH * 2) + sub * 16) =
          make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    } else {
      const float* scale = is_v ? a.v_scale : a.k_scale;
      const float inv = scale ? 1.0f / scale[kh] : 1.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = to_e4m3_range(y[j] * inv);
      *reinterpret_cast<uint2*>(pool + row * DH + sub * 8) = make_uint2(pack_e4m3x4(y[0], y[1], y[2], y[3]), pack_e4m3x4(y[4], y[5], y[6], y[7]));
    }
  }
}

hipError_t launch_qk_norm_rope(const QkArgs& a, uint32_t head_dim, double theta, hipStream_t st) {
  if (a.n_tokens == 0) return hipSuccess;
  RopeTurns turns = {};
  for (uint32_t i = 0; a.rope && i < head_dim / 2; ++i)
    turns.t[i] = std::pow(theta, -2.0 * i / head_dim) * 0.15915494309189533577;      // 1 / 2 pi
  const uint32_t heads = a.q_heads + a.kv_heads * (a.cache_type ? 2u : 1u), per = 512 / head_dim, groups = (heads + per - 1) / per;
  const uint32_t parts = std::max(1u, std::min(groups, 4096u / a.n_tokens));
  const uint32_t wgs = (uint32_t)(((uint64_t)a.n_tokens * parts + 3) / 4);
  if (head_dim == 128) qk_norm_rope_kernel<128><<<wgs, 256, 0, st>>>(a, turns, parts);
  else qk_norm_rope_kernel<64><<<wgs, 256, 0, st>>>(a, turns, parts);
  return hipGetLastError();
}

}  // namespace qzo
