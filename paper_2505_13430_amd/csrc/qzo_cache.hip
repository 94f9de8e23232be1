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

// Slot of position `at` in block `id`; none in a block that the pool has not: shifted, such an id could end at another block's slot.
__device__ __forceinline__ int32_t slot_of(const CachePlanArgs& a, int32_t id, int32_t at) {
  return (uint32_t)id < a.n_blocks ? (int32_t)(((uint32_t)id << a.block_shift) + ((uint32_t)at & ((1u << a.block_shift) - 1u))) : -1;
}

// One workgroup, a sequence (or several) per thread.  What sequence i gives back (ended), takes and adds is summed over the
// sequences before it; the sums stay in the LDS, where blocks given back, and the blocks and tokens of long prompts, find their
// sequence by bisection and are spread over all threads.  Every input is read before the first output is written (lengths
// may be cached, after may be before), and no output of this launch is read back: a taken block is found in the free list or
// in the row of the sequence that gives it back, neither of which changes below the stack's old height.
// Latency is all there is to it: lengths, sums, free list, stores.  The block that a sequence's next token falls into is
// loaded beside the lengths.  8 sequences 3.8 us, 1000 6.4, 300 with prompts of 801 tokens 10.4 with the second launch.
// with_slots: slots and positions too (few tokens); else cache_slots_kernel follows.
constexpr uint32_t PLAN_THREADS = 1024, PLAN_FEW = 4;      // a thread itself sees to that many tokens, and their blocks
__global__ __launch_bounds__(PLAN_THREADS) void cache_plan_kernel(CachePlanArgs a, uint32_t with_slots) {
  extern __shared__ int32_t prefix[];
  int32_t* const back = prefix;                    // [n_seq] blocks given back before sequence i
  int32_t* const take = prefix + a.n_seq;          // [n_seq] blocks taken before it
  int32_t* const start = prefix + 2 * a.n_seq;     // [n_seq] tokens added before it
  int32_t* const old_len = prefix + 3 * a.n_seq;   // [n_seq]
  __shared__ uint32_t wave_sums[3][PLAN_THREADS / 64];
  __shared__ float wave_sizes[3][PLAN_THREADS / 64];
  __shared__ uint32_t flags;                       // 1: wrong, 2: a row too short, 4: a sequence of more than PLAN_FEW tokens
  const uint32_t tid = threadIdx.x, shift = a.block_shift;
  const int32_t mask = (1 << shift) - 1;
  const int64_t room = (int64_t)a.max_blocks << shift;
  const uint32_t per = (a.n_seq + PLAN_THREADS - 1) / PLAN_THREADS, first = min(tid * per, a.n_seq), last = min(first + per, a.n_seq);
  if (tid == 0) flags = 0;
  __syncthreads();
  const int32_t n_free = a.before->n_free;
  auto blocks = [&](int64_t tokens) { return (tokens + mask) >> shift; };
  int64_t sum[3] = {0, 0, 0};
  uint32_t seen = n_free < 0 || (uint32_t)n_free > a.n_blocks ? 1u : 0u;
  int32_t open = 0;                                // per = 1: the block that holds the sequence's last token
  const int32_t add0 = first < last ? a.added[first] : 0;      // a thread's first sequence, mostly its only one
  auto added = [&](uint32_t i) { return i == first ? add0 : a.added[i]; };
  for (uint32_t i = first; i < last; ++i) {
    const int32_t have = a.cached[i], add = added(i);
    if (have < 0) seen |= 1u;
    else if (have > room || (add > 0 && (int64_t)have + add > room)) seen |= 2u;
    else if (per == 1 && have > 0) open = a.tables[(uint64_t)i * a.max_blocks + (uint32_t)((have - 1) >> shift)];
    if (add > (int32_t)PLAN_FEW) seen |= 4u;
    sum[0] += add < 0 ? blocks(have) : 0;
    sum[1] += add < 0 ? 0 : blocks((int64_t)have + add) - blocks(have);
    sum[2] += add < 0 ? 0 : add;
    old_len[i] = have;
  }
  if (seen) atomicOr(&flags, seen);
  // exclusive sums over the threads, in 32 bits; whether 32 bits hold them is told by sums of floats (a whole plan has totals
  // below 2^31, what a float misses of them is far below 2^31 too)
  uint32_t run[3];
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const uint32_t v = (uint32_t)sum[j], upto = lane_scan(v);
    const float size = lane_scan((float)sum[j]);
    if ((tid & 63u) == 63u) { wave_sums[j][tid >> 6] = upto; wave_sizes[j][tid >> 6] = size; }
    run[j] = upto - v;
  }
  __syncthreads();
  uint32_t total[3];
  bool fits[3];
  constexpr uint32_t N = PLAN_THREADS / 64;
  const uint32_t lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const uint32_t v = lane < N ? wave_sums[j][lane] : 0u, upto = lane_scan(v);
    const float size = lane_scan(lane < N ? wave_sizes[j][lane] : 0.0f);
    run[j] += (uint32_t)__builtin_amdgcn_readlane((int)(upto - v), (int)wave);
    total[j] = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    fits[j] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(size), 63)) < 3e9f && total[j] < 0x80000000u;
  }
  const uint32_t flag = flags;
  int32_t status = QZO_OK;
  if (flag & 1u) status = QZO_ERR_ARG;
  else if ((flag & 2u) || !fits[2] || total[2] > a.max_tokens) status = QZO_ERR_SHAPE;
  else if (!fits[0] || (uint32_t)n_free + total[0] > a.n_blocks) status = QZO_ERR_ARG;        // more blocks than there are
  else if (!fits[1] || total[1] > (uint32_t)n_free + total[0]) status = QZO_ERR_WORKSPACE;
  const bool ok = status == QZO_OK;
  const int32_t n_back = ok ? (int32_t)total[0] : 0, n_take = ok ? (int32_t)total[1] : 0, n_tok = ok ? (int32_t)total[2] : 0;
  {
    uint32_t b = run[0], k = run[1], t = run[2];
    for (uint32_t i = first; i < last; ++i) {
      const int32_t have = old_len[i], add = added(i);
      back[i] = (int32_t)b; take[i] = (int32_t)k; start[i] = (int32_t)t;
      a.lengths[i] = !ok ? have : add < 0 ? 0 : have + add;
      a.starts[i] = ok ? (int32_t)t : 0;
      if (add < 0) b += (uint32_t)blocks(have);
      else { k += (uint32_t)(blocks((int64_t)have + add) - blocks(have)); t += (uint32_t)add; }
    }
  }
  if (tid == 0) {
    a.starts[a.n_seq] = n_tok;
    *a.after = qzo_cache_state{n_free + n_back - n_take, n_tok, status, n_take};
  }
  if (!ok) {
    for (uint32_t t = tid; with_slots && t < a.max_tokens; t += PLAN_THREADS) { a.slots[t] = -1; a.positions[t] = 0; }
    return;
  }
  __syncthreads();
  auto given = [&](int32_t r) {                  // r-th block given back
    const uint32_t s = last_not_above(back, a.n_seq, r);
    return a.tables[(uint64_t)s * a.max_blocks + (uint32_t)(r - back[s])];
  };
  auto taken = [&](int32_t k) {                  // k-th block taken: those given back lie on top of the free ones
    return k < n_back ? given(n_back - 1 - k) : a.free[n_free - 1 - (k - n_back)];
  };
  // a sequence's block number j, one that it held or one that it takes
  auto block_of = [&](uint32_t i, int32_t j, int32_t held) { return j < held ? a.tables[(uint64_t)i * a.max_blocks + (uint32_t)j] : taken(take[i] + j - held); };
  if (!(flag & 4u)) {
    for (uint32_t i = first; i < last; ++i) {
      const int32_t have = old_len[i], add = added(i), held = (int32_t)blocks(have);
      int32_t number = -1, id = 0;
      for (int32_t x = 0; x < add; ++x) {
        const int32_t at = have + x, j = at >> shift;
        if (j != number) {
          id = per == 1 && j == held - 1 ? open : block_of(i, j, held);
          number = j;
          if (j >= held) a.tables[(uint64_t)i * a.max_blocks + (uint32_t)j] = id;
        }
        if (with_slots) { a.slots[start[i] + x] = slot_of(a, id, at); a.positions[start[i] + x] = at; }
      }
    }
  } else {
#pragma unroll 4
    for (int32_t k = (int32_t)tid; k < n_take; k += PLAN_THREADS) {
      const uint32_t s = last_not_above(take, a.n_seq, k);
      a.tables[(uint64_t)s * a.max_blocks + (uint32_t)blocks(old_len[s]) + (uint32_t)(k - take[s])] = taken(k);
    }
    for (int32_t t = (int32_t)tid; with_slots && t < n_tok; t += PLAN_THREADS) {
      const uint32_t s = last_not_above(start, a.n_seq, t);
      const int32_t at = old_len[s] + t - start[s];
      a.slots[t] = slot_of(a, block_of(s, at >> shift, (int32_t)blocks(old_len[s])), at);
      a.positions[t] = at;
    }
  }
  // (threads that had the least to do so far)
  for (int32_t r = (int32_t)(PLAN_THREADS - 1 - tid); r < n_back - n_take; r += PLAN_THREADS) a.free[n_free + r] = given(r);
  for (uint32_t t = (uint32_t)n_tok + tid; with_slots && t < a.max_tokens; t += PLAN_THREADS) { a.slots[t] = -1; a.positions[t] = 0; }
}

// Slots and positions of many tokens, from what cache_plan_kernel left.
__global__ __launch_bounds__(256) void cache_slots_kernel(CachePlanArgs a) {
  extern __shared__ int32_t prefix[];
  for (uint32_t i = threadIdx.x; i <= a.n_seq; i += 256) prefix[i] = a.starts[i];
  __syncthreads();
  const int32_t n_tok = prefix[a.n_seq];
  for (uint32_t t = blockIdx.x * 256u + threadIdx.x; t < a.max_tokens; t += gridDim.x * 256u) {
    int32_t slot = -1, at = 0;
    if ((int32_t)t < n_tok) {
      const uint32_t s = last_not_above(prefix, a.n_seq, (int32_t)t);
      at = a.lengths[s] - (prefix[s + 1] - (int32_t)t);
      slot = slot_of(a, a.tables[(uint64_t)s * a.max_blocks + (uint32_t)(at >> a.block_shift)], at);
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
  cache_slots_kernel<<<std::min<uint32_t>((a.max_tokens + 255) / 256, 2048u), 256, (a.n_seq + 1) * 4u, st>>>(a);
  return hipGetLastError();
}

// ------------------------------------------------------------ heads of q and k ----
// y = R(position) (x / sqrt(mean x^2 + eps) * gain), head by head: RMSNorm over the head's DH features, then the pairs
// (i, i + DH/2) turned by position * theta^(-2i/DH).  Everything between the load and the one rounding at the store is
// fp32; the angle is formed in double as a number of turns (position times theta^(-2i/DH) / 2 pi) and only its fraction
// goes to fp32, so that far positions lose nothing.
// DH/8 lanes hold a head, eight features each; a wavefront takes 64 / (DH/8) heads at a time and walks over its share of
// the token's heads with the same angles.
//
// Memory counts, and how much of it is on its way: a wavefront loads its next heads before it works on the ones it has, and a
// token is spread over as many wavefronts as it takes to have QK_WAVES of them (2500 tokens, 120 heads of 128, with 4096 / 8192 /
// 16384 / 24576 / 32768 / 65536: 44 / 37 / 35 / 34 / 34 / 40 us).  The cosine and sine of a pair are computed once per
// wavefront, by one lane, and handed out through the LDS (each lane its own eight: 41 us).  One token 2.5 us; 16 x 512 tokens,
// q and k of 32 heads of 128: 53 us, 5.0 TB/s read and written, as a copy of 2 GiB (4.9); with an e4m3 cache, 7001 tokens, 64
// and 8 heads of 64, 30 us, 4.6 TB/s.

// Values of the lanes of a head (16, or 8): their sum; that of the lane half a head away.  Exchanges within rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
template <int DH>
__device__ __forceinline__ float sum_of_head(float v) {
  v += from_lane<0xB1>(v);                      // quad_perm 1,0,3,2
  v += from_lane<0x4E>(v);                      // quad_perm 2,3,0,1
  v += from_lane<0x141>(v);                     // row_half_mirror: the other four of eight
  if (DH == 128) v += from_lane<0x140>(v);      // row_mirror: the other eight of sixteen
  return v;
}
template <int DH>
__device__ __forceinline__ float half_a_head_away(float v) {
  if (DH == 128) return from_lane<0x128>(v);              // row_ror:8
  return from_lane<0x1B>(from_lane<0x141>(v));            // mirrored in eight, then in four: four away
}

template <int DH>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a, RopeTurns turns, uint32_t parts) {
  constexpr uint32_t LANES = DH / 8, HEADS = 64 / LANES;
  const uint32_t lane = threadIdx.x & 63u, sub = lane % LANES;
  const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4u + (threadIdx.x >> 6))), t = w / parts, part = w % parts;
  if (t >= a.n_tokens) return;
  int32_t slot = 0;
  if (a.slots) {
    slot = a.slots[t];
    if (slot < 0 || (uint32_t)slot >= a.n_slots) return;
  }
  const uint32_t n_qk = a.q_heads + a.kv_heads, heads = n_qk + (a.cache_type ? a.kv_heads : 0u), turn = parts * HEADS;
  const bf16_t* const row = a.qkv + (uint64_t)t * a.ld_qkv + sub * 8;
  const uint32_t h0 = part * HEADS + lane / LANES;
  // all lanes of a wavefront make the same number of turns; a head beyond the last is read as the last and not written
  const uint32_t n_turns = (heads - part * HEADS + turn - 1) / turn;
  auto load = [&](uint32_t i) { return *reinterpret_cast<const uint4*>(row + (uint64_t)min(h0 + i * turn, heads - 1u) * DH); };
  uint4 raw = load(0);
  uint4 q_gain = make_uint4(0u, 0u, 0u, 0u), k_gain = q_gain;
  if (a.q_gain) q_gain = *reinterpret_cast<const uint4*>(a.q_gain + sub * 8);
  if (a.k_gain) k_gain = *reinterpret_cast<const uint4*>(a.k_gain + sub * 8);
  const int32_t at = a.positions ? a.positions[t] : (int32_t)((t % a.pass_stride) % a.seq);
  // a pair's angle per lane, all eight of a lane's features by way of the LDS
  __shared__ __attribute__((aligned(16))) float2 angles[4][DH / 2];
  float c[8], s[8];
  if (a.rope) {
    float2* const mine = angles[threadIdx.x >> 6];
    if (lane < DH / 2) {
      const double rev = (double)at * turns.t[lane];
      float2 cs;
      sincospif(2.0f * (float)(rev - rint(rev)), &cs.y, &cs.x);
      mine[lane] = cs;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 cs = mine[(sub * 8 + j) % (DH / 2)];
      c[j] = cs.x;
      s[j] = sub < LANES / 2 ? -cs.y : cs.y;
    }
  }
  const uint64_t slot_row = ((uint64_t)((uint32_t)slot >> a.block_shift) * a.kv_heads << a.block_shift) + ((uint32_t)slot & ((1u << a.block_shift) - 1u));
  for (uint32_t i = 0; i < n_turns; ++i) {
    const uint4 now = raw;
    if (i + 1 < n_turns) raw = load(i + 1);
    const uint32_t h = h0 + i * turn, r[4] = {now.x, now.y, now.z, now.w};
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(r[j] << 16);
      x[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
    const bool is_q = h < a.q_heads, is_v = h >= n_qk;
    if (a.q_gain || a.k_gain) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = __builtin_fmaf(x[j], x[j], ss);
      const float inv = __builtin_amdgcn_rsqf(sum_of_head<DH>(ss) * (1.0f / DH) + a.eps);
      if (is_q ? a.q_gain != nullptr : !is_v && a.k_gain) {
        const uint32_t g[4] = {is_q ? q_gain.x : k_gain.x, is_q ? q_gain.y : k_gain.y, is_q ? q_gain.z : k_gain.z, is_q ? q_gain.w : k_gain.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[2 * j] *= inv * __uint_as_float(g[j] << 16);
          x[2 * j + 1] *= inv * __uint_as_float(g[j] & 0xffff0000u);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float other = half_a_head_away<DH>(x[j]);
      y[j] = is_v || !a.rope ? x[j] : __builtin_fmaf(other, s[j], x[j] * c[j]);
    }
    if (h >= heads) continue;
    if (is_q || !a.cache_type) {
      *reinterpret_cast<uint4*>(a.out + (uint64_t)t * a.ld_out + (uint64_t)h * DH + sub * 8) =
          make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
      continue;
    }
    const uint32_t kh = h - (is_v ? n_qk : a.q_heads);
    const uint64_t at_row = slot_row + ((uint64_t)kh << a.block_shift);
    unsigned char* pool = (unsigned char*)(is_v ? a.v : a.k);
    if (a.cache_type == 1) {
      *reinterpret_cast<uint4*>(pool + at_row * (DH * 2) + sub * 16) =
          make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    } else {
      const float* scale = is_v ? a.v_scale : a.k_scale;
      const float inv = scale ? 1.0f / scale[kh] : 1.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = to_e4m3_range(y[j] * inv);
      *reinterpret_cast<uint2*>(pool + at_row * DH + sub * 8) = make_uint2(pack_e4m3x4(y[0], y[1], y[2], y[3]), pack_e4m3x4(y[4], y[5], y[6], y[7]));
    }
  }
}

constexpr uint32_t QK_WAVES = 24576;
hipError_t launch_qk_norm_rope(const QkArgs& a, uint32_t head_dim, double theta, hipStream_t st) {
  if (a.n_tokens == 0) return hipSuccess;
  RopeTurns turns = {};
  for (uint32_t i = 0; a.rope && i < head_dim / 2; ++i)
    turns.t[i] = std::pow(theta, -2.0 * i / head_dim) * 0.15915494309189533577;      // 1 / 2 pi
  const uint32_t heads = a.q_heads + a.kv_heads * (a.cache_type ? 2u : 1u), per = 512 / head_dim, groups = (heads + per - 1) / per;
  const uint32_t parts = std::max(1u, std::min(groups, QK_WAVES / a.n_tokens));
  const uint64_t wgs = ((uint64_t)a.n_tokens * parts + 3) / 4;
  if (head_dim == 128) qk_norm_rope_kernel<128><<<(uint32_t)wgs, 256, 0, st>>>(a, turns, parts);
  else qk_norm_rope_kernel<64><<<(uint32_t)wgs, 256, 0, st>>>(a, turns, parts);
  return hipGetLastError();
}

}  // namespace qzo
