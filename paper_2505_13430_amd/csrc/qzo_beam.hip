// The next beams of every prompt: of all continuations of its beams by a token the best ones, and the beams' states reordered with them.
//
//   total(b, v) = score(b) + x(b, v) - lse(b), lse(b) = log sum_v e^x(b, v);  key = total, or total / count^alpha.
// Within a beam the order is that of the logits, so a row's best tokens are found without its lse, in the same pass that sums it up.
#include <algorithm>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {
namespace {

constexpr uint32_t PART_THREADS = 256, PART_WAVES = PART_THREADS / 64, LANE = 16, TILE = 64 * LANE;      // logits of a lane and of a wavefront at a time
constexpr uint32_t MAX_PARTS = 64, MAX_SPAN = 65536;          // a logit's place in a part is 16 bits
constexpr uint32_t MERGE_THREADS = 1024, MERGE_WAVES = MERGE_THREADS / 64;

// Highest value of the wavefront's lanes, 0 the lowest there is.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t higher(uint32_t v) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false)); }
__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
  v = higher<0x111, 0xf>(v);
  v = higher<0x112, 0xf>(v);
  v = higher<0x114, 0xf>(v);
  v = higher<0x118, 0xf>(v);
  v = higher<0x142, 0xa>(v);
  v = higher<0x143, 0xc>(v);
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// e^d, d <= 0.  The product with log2(e) is taken in two parts: what it is off by would be off in every term with that logit.
__device__ __forceinline__ float exp_of(float d) {
  const float LOG2E = 1.44269502162933349609375f, LOG2E_REST = 1.92596299112661746887e-8f, LN2 = 0.693147180559945f;
  const float y = d * LOG2E, rest = __builtin_fmaf(d, LOG2E_REST, __builtin_fmaf(d, LOG2E, -y));
  const float e = __builtin_amdgcn_exp2f(y);
  return __builtin_fmaf(e, rest * LN2, e);
}

// A logit as 16 bits that order as the numbers do; 0: none (NaN and infinities).
__device__ __forceinline__ uint32_t order_of(uint32_t bits) {
  if ((bits & 0x7f80u) == 0x7f80u) return 0u;
  if (bits == 0x8000u) bits = 0u;              // -0
  return (bits & 0x8000u) ? (~bits & 0xffffu) : (bits | 0x8000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __uint_as_float(((order & 0x8000u) ? order & 0x7fffu : ~order & 0xffffu) << 16);
}

// ---- a part of a row: its best tokens, its maximum and its sum
// A wavefront's part, TILE logits at a time.  The best ones so far are in its lanes, in order; a tile with none above the last of them
// is done with a maximum of its keys (the logit's order above, the place from behind below: no two are equal).
__global__ __launch_bounds__(PART_THREADS) void beam_parts_kernel(BeamArgs a) {
  const uint32_t lane = threadIdx.x & 63u;
  const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * PART_WAVES + (threadIdx.x >> 6))), row = w / a.parts, part = w % a.parts;
  if (row >= a.n_rows || a.ended[row] || !(a.scores[row] > -INFINITY)) return;
  const uint32_t v0 = part * a.span, v1 = min(v0 + a.span, a.vocab);
  const bf16_t* const x = a.logits + (uint64_t)row * a.ld;
  // 16-byte pieces as they lie in memory: the first may begin before the part, the last end behind it
  const uint32_t skew = (uint32_t)((uintptr_t)(x + v0) & 15u) / 2u;
  uint32_t best = 0, bound = 0;
  float m = -INFINITY;
  double sum = 0.0;
  for (int64_t t0 = (int64_t)v0 - skew; t0 < (int64_t)v1; t0 += TILE) {
    uint32_t key[LANE], top = 0;
#pragma unroll
    for (uint32_t u = 0; u < LANE / 8; ++u) {
      const int64_t v = t0 + u * 512 + lane * 8u;
      uint32_t bits[8];
      if (v >= (int64_t)v0 && v + 8 <= (int64_t)v1) {
        const uint4 q = *reinterpret_cast<const uint4*>(x + v);
        const uint32_t d[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) bits[j] = d[j / 2] >> 16 * (j & 1) & 0xffffu;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) bits[j] = v + j >= (int64_t)v0 && v + j < (int64_t)v1 ? x[v + j] : 0xff80u;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t o = order_of(bits[j]);
        key[u * 8 + j] = o ? o << 16 | (MAX_SPAN - 1u - (uint32_t)(v + j - v0)) : 0u;
        top = max(top, key[u * 8 + j]);
      }
    }
    if (top) {
      const float tile_top = value_of(top >> 16), m2 = fmaxf(m, tile_top);
      float s = 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < LANE; ++u) s += key[u] ? exp_of(value_of(key[u] >> 16) - m2) : 0.0f;
      sum = (m > -INFINITY ? sum * (double)exp_of(m - m2) : 0.0) + (double)s;
      m = m2;
    }
    while (__any(top > bound)) {
      const uint32_t got = wave_top(top);
      const uint32_t before = (uint32_t)__shfl_up((int)best, 1, 64);
      best = best > got ? best : lane == 0 || before > got ? got : before;
      bound = (uint32_t)__builtin_amdgcn_readlane((int)best, (int)a.width - 1);
      if (top == got) {
        top = 0;
#pragma unroll
        for (uint32_t u = 0; u < LANE; ++u) top = max(top, key[u] < got ? key[u] : 0u);
      }
    }
  }
  if (lane < a.width) a.best[(uint64_t)w * a.width + lane] = best;
  float all_m = m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) all_m = fmaxf(all_m, __shfl_xor(all_m, o, 64));
  double all = m > -INFINITY ? sum * (double)exp_of(m - all_m) : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o, 64);
  if (lane == 0) a.sums[w] = BeamSum{all, all_m, 0};
}

// A candidate: the higher key first, then the lower place (beam and token).
struct Candidate {
  double key = -INFINITY;
  uint32_t place = ~0u;
  __device__ __forceinline__ bool before(const Candidate& o) const { return key > o.key || (key == o.key && place < o.place); }
};
__device__ __forceinline__ Candidate wave_first(Candidate c) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    Candidate d;
    d.key = __shfl_xor(c.key, o, 64);
    d.place = (uint32_t)__shfl_xor((int)c.place, o, 64);
    if (d.before(c)) c = d;
  }
  return c;
}

// ---- a prompt's beams out of its parts'
__global__ __launch_bounds__(MERGE_THREADS) void beam_merge_kernel(BeamArgs a) {
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t W = a.width, r0 = blockIdx.x * W;
  __shared__ double lse[BEAM_MAX_WIDTH], score[BEAM_MAX_WIDTH], factor[BEAM_MAX_WIDTH];        // factor: what a beam's totals are divided by
  __shared__ int32_t count[BEAM_MAX_WIDTH], parent[BEAM_MAX_WIDTH], token[BEAM_MAX_WIDTH];
  __shared__ uint32_t kind[BEAM_MAX_WIDTH];                                                     // 0: none, 1: goes on, 2: has ended
  __shared__ double found_key[MERGE_WAVES][BEAM_MAX_WIDTH];
  __shared__ uint32_t found_place[MERGE_WAVES][BEAM_MAX_WIDTH];
  __shared__ uint32_t last;
  for (uint32_t b = wave; b < W; b += MERGE_WAVES) {
    const float s = a.scores[r0 + b];
    const uint32_t k = !(s > -INFINITY) ? 0u : a.ended[r0 + b] ? 2u : 1u;
    if (lane == 0) {
      const int32_t c = max(0, a.counts[r0 + b]);
      kind[b] = k; score[b] = (double)s; count[b] = c;
      factor[b] = a.penalty == 0.0 ? 1.0 : pow((double)max(1, k == 1u ? c + (c < INT32_MAX) : c), a.penalty);
    }
    if (k != 1u) continue;
    BeamSum p = {0.0, -INFINITY, 0};
    if (lane < a.parts) p = a.sums[(uint64_t)(r0 + b) * a.parts + lane];
    float m = p.top;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    double n = p.top > -INFINITY ? p.sum * (double)exp_of(p.top - m) : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    if (lane == 0) lse[b] = log(n) + (double)m;
  }
  __syncthreads();
  // every wavefront the best of its lists (a part of a row, in order), then the first one the best of theirs
  const uint32_t lists = W * a.parts;
  auto total_of = [&](uint32_t b, uint32_t v, float x) { return kind[b] == 2u ? score[b] : ((double)x - lse[b]) + score[b]; };
  auto candidate = [&](uint32_t list, uint32_t at) {
    Candidate c;
    const uint32_t b = list / a.parts, part = list % a.parts;
    if (kind[b] == 2u) {
      if (part == 0 && at == 0) { c.key = score[b] / factor[b]; c.place = b * a.vocab + (uint32_t)max(a.end_token, 0); }
    } else if (kind[b] == 1u && at < W) {
      const uint32_t key = a.best[((uint64_t)(r0 + b) * a.parts + part) * W + at];
      if (key) {
        const uint32_t v = part * a.span + (MAX_SPAN - 1u - (key & 0xffffu));
        const double t = total_of(b, v, value_of(key >> 16));
        c.key = a.penalty == 0.0 ? t : t / factor[b];
        c.place = b * a.vocab + v;
      }
    }
    return c;
  };
  constexpr uint32_t OWN = BEAM_MAX_WIDTH * MAX_PARTS / MERGE_THREADS;          // lists of a thread
  {
    Candidate head[OWN], mine;
    uint32_t at[OWN];
    const uint32_t n_own = (lists + MERGE_THREADS - 1) / MERGE_THREADS;
#pragma unroll
    for (uint32_t u = 0; u < OWN; ++u) {
      at[u] = 0;
      if (u < n_own && tid + u * MERGE_THREADS < lists) head[u] = candidate(tid + u * MERGE_THREADS, 0);
      if (head[u].before(mine)) mine = head[u];
    }
    for (uint32_t r = 0; r < W; ++r) {
      const Candidate c = wave_first(mine);
      if (lane == 0) { found_key[wave][r] = c.key; found_place[wave][r] = c.place; }
      if (c.place == ~0u) continue;
      if (mine.place == c.place) {
        mine = Candidate{};
#pragma unroll
        for (uint32_t u = 0; u < OWN; ++u) {
          if (u < n_own && head[u].place == c.place) head[u] = candidate(tid + u * MERGE_THREADS, ++at[u]);
          if (head[u].before(mine)) mine = head[u];
        }
      }
    }
  }
  __syncthreads();
  if (wave == 0) {
    uint32_t at = 0;
    Candidate mine;
    if (lane < MERGE_WAVES) { mine.key = found_key[lane][0]; mine.place = found_place[lane][0]; }
    for (uint32_t r = 0; r < W; ++r) {
      const Candidate c = wave_first(mine);
      const bool some = c.place != ~0u;
      if (lane == 0) {
        parent[r] = some ? (int32_t)(c.place / a.vocab) : -1;
        token[r] = some ? (int32_t)(c.place % a.vocab) : -1;
      }
      if (some && mine.place == c.place) {
        ++at;
        mine = Candidate{};
        if (at < W) { mine.key = found_key[lane][at]; mine.place = found_place[lane][at]; }
      }
    }
  }
  __syncthreads();
  // ---- states
  if (tid < W) {
    const int32_t b = parent[tid], v = token[tid];
    const uint32_t r = r0 + tid;
    float s = -INFINITY;
    int32_t n = 0, ended = 1;
    if (b >= 0) {
      const bool was = kind[b] == 2u;
      s = (float)total_of((uint32_t)b, (uint32_t)v, was ? 0.0f : __uint_as_float((uint32_t)a.logits[(uint64_t)(r0 + b) * a.ld + v] << 16));
      n = was || count[b] == INT32_MAX ? count[b] : count[b] + 1;
      ended = was || v == a.end_token;
    }
    a.scores[r] = s;
    a.counts[r] = n;
    a.ended[r] = ended;
    a.parents[r] = b < 0 ? -1 : (int32_t)(r0 + b);
    a.chosen[r] = v;
    a.added[r] = !ended;
  }
  // histories, some columns of all rows at a time: read, then written
  uint32_t longest = 0;
  for (uint32_t b = 0; b < W; ++b)
    if (parent[b] >= 0) longest = max(longest, min((uint32_t)count[parent[b]] + 1u, a.max_history));
  constexpr uint32_t HELD = 8;
  const uint32_t columns = MERGE_THREADS * HELD / W;
  for (uint32_t c0 = 0; c0 < longest; c0 += columns) {
    const uint32_t n = min(columns, longest - c0);
    int32_t held[HELD];
#pragma unroll
    for (uint32_t u = 0; u < HELD; ++u) {
      const uint32_t e = u * MERGE_THREADS + tid, i = e / n, c = c0 + e % n;
      if (e >= n * W || parent[i] < 0) continue;
      const uint32_t b = (uint32_t)parent[i];
      if (c < (uint32_t)count[b]) held[u] = a.history[(uint64_t)(r0 + b) * a.max_history + c];
      else if (c == (uint32_t)count[b] && kind[b] == 1u) held[u] = token[i];
    }
    __syncthreads();
#pragma unroll
    for (uint32_t u = 0; u < HELD; ++u) {
      const uint32_t e = u * MERGE_THREADS + tid, i = e / n, c = c0 + e % n;
      if (e >= n * W || parent[i] < 0) continue;
      const uint32_t b = (uint32_t)parent[i];
      if (c < (uint32_t)count[b] || (c == (uint32_t)count[b] && kind[b] == 1u)) a.history[(uint64_t)(r0 + i) * a.max_history + c] = held[u];
    }
    __syncthreads();
  }
}

// ---- the tokens of the beams that go on, one behind the other
__global__ __launch_bounds__(MERGE_THREADS) void beam_pack_kernel(BeamArgs a) {
  const uint32_t tid = threadIdx.x;
  __shared__ uint32_t red[MERGE_WAVES];
  uint32_t before = 0;
  for (uint32_t j0 = 0; j0 < a.n_rows; j0 += MERGE_THREADS) {
    const uint32_t j = j0 + tid, on = j < a.n_rows && a.added[j], upto = lane_scan(on);
    __syncthreads();
    if ((tid & 63u) == 63u) red[tid >> 6] = upto;
    __syncthreads();
    uint32_t at = before, all = 0;
    for (uint32_t w = 0; w < MERGE_WAVES; ++w) {
      if (w < (tid >> 6)) at += red[w];
      all += red[w];
    }
    if (on) a.tokens[at + upto - 1u] = a.chosen[j];
    before += all;
  }
  for (uint32_t j = before + tid; j < a.n_rows; j += MERGE_THREADS) a.tokens[j] = 0;
}

// Parts of a row: enough wavefronts for the chip, tiles enough for each.
constexpr uint32_t WANTED_WAVES = 4096;
void cut(uint32_t n_rows, uint32_t vocab, uint32_t* parts, uint32_t* span) {
  uint32_t p = std::min((vocab + TILE - 1) / TILE, std::max(1u, WANTED_WAVES / n_rows));
  p = std::min(std::max(p, (vocab + MAX_SPAN - 1) / MAX_SPAN), MAX_PARTS);
  *span = std::min(((vocab + p - 1) / p + 7) / 8 * 8, MAX_SPAN);
  *parts = (vocab + *span - 1) / *span;
}
uint64_t up16(uint64_t bytes) { return (bytes + 15) & ~15ull; }

}  // namespace

uint64_t beam_select_scratch(uint32_t n_rows, uint32_t width, uint32_t vocab) {
  uint32_t parts, span;
  cut(n_rows, vocab, &parts, &span);
  return up16((uint64_t)n_rows * parts * sizeof(BeamSum)) + up16(4ull * n_rows * parts * width);
}

hipError_t launch_beam_select(BeamArgs a, void* scratch, hipStream_t st) {
  cut(a.n_rows, a.vocab, &a.parts, &a.span);
  a.sums = (BeamSum*)scratch;
  a.best = (uint32_t*)((char*)scratch + up16((uint64_t)a.n_rows * a.parts * sizeof(BeamSum)));
  const uint64_t waves = (uint64_t)a.n_rows * a.parts;
  beam_parts_kernel<<<(uint32_t)((waves + PART_WAVES - 1) / PART_WAVES), PART_THREADS, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  beam_merge_kernel<<<a.n_rows / a.width, MERGE_THREADS, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  beam_pack_kernel<<<1, MERGE_THREADS, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace qzo
