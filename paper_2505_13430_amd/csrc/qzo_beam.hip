// The next beams of every prompt: of all continuations of its beams by a token the best ones, and the beams' states reordered with them.
//
//   total(b, v) = score(b) + x(b, v) - lse(b), lse(b) = log sum_v e^x(b, v);  key = total, or total / count^alpha.
// Within a beam the order is that of the logits, so a row's best tokens are found without its lse, in the same pass that sums it up.
#include <algorithm>
#include <type_traits>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {
namespace {

constexpr uint32_t THREADS = 256, WAVES = THREADS / 64, LANE = 16, TILE = 64 * LANE;      // logits of a lane and of a wavefront at a time
constexpr uint32_t MAX_PARTS = 64, MAX_SPAN = 65536;          // a logit's place in a part is 16 bits
constexpr double LN2 = 0.693147180559945309417;
constexpr float LOG2E = 1.44269504088896f, HIGHEST = 8.0f, LARGE = 32768.0f;

// Highest and lowest value of the wavefront's lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t higher(uint32_t v) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false)); }
__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
  v = higher<0x111, 0xf>(v);                    // row_shr:1, 2, 4, 8
  v = higher<0x112, 0xf>(v);
  v = higher<0x114, 0xf>(v);
  v = higher<0x118, 0xf>(v);
  v = higher<0x142, 0xa>(v);                    // row_bcast:15
  v = higher<0x143, 0xc>(v);                    // row_bcast:31
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
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
__device__ __forceinline__ float low_half(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_half(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// Sum over the wavefront's lanes, in the order of lane_scan.
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lane(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, false), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_total(double v) {
  v += from_lane<0x111, 0xf>(v);
  v += from_lane<0x112, 0xf>(v);
  v += from_lane<0x114, 0xf>(v);
  v += from_lane<0x118, 0xf>(v);
  v += from_lane<0x142, 0xa>(v);
  v += from_lane<0x143, 0xc>(v);
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63));
}
// A float as 32 bits that order as the numbers do, 0 below all, and back.
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t b = __float_as_uint(f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }

// Words for another workgroup, on any XCD: stored through the L2, loaded past it.
__device__ __forceinline__ void share_out(uint32_t* p, uint32_t x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t shared_in(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void share_out(double* p, double x) { __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double shared_in(const double* p) { return __builtin_bit_cast(double, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)); }
// Whether this workgroup is the last of `all` to come here; what it and the others shared out before is there then.
__device__ __forceinline__ bool last_of(uint32_t* counter, uint32_t all, uint32_t* flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last = atomicAdd(counter, 1u) + 1u == all;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  return *flag != 0u;
}

// ---- a part of a row: its best tokens and its sum
// A wavefront's part, TILE logits at a time, the next ones on their way.  Memory is what is to count, so a logit costs few instructions: half a
// maximum, and 2^(x log2(e) - c) into the sum.  c stands for the part's maximum m; it is the first tile's, or a later one's that is
// 2^HIGHEST above it, a float that the sum is relative to exactly: the old sum is scaled by 2^(c - c2) in 64 bits, so that c's rounding is in
// no result.  What is off, of a term near the maximum: log2(e) as a float (1.3e-8 of x - m), the product's rounding (2^-22 where the exponent is 4 to 8, 2.8 x
// 2^-24 of the term), the exponential's (one ulp), a lane's sum of 16; at most some 16 x 2^-24, far less for a sum over many, whose
// terms' roundings differ.  (With HIGHEST 60 the product's rounding is 2^-19 of a term, and 480 rows of 99991 or 4 of 32000 take as long.)
//   A tile whose sum or maximum tells of a NaN or an infinity is gone through again, logit by logit; so is every tile while the reference is LARGE:
// x log2(e) and c are rounded to more than 2^-9 there (to more than the exponents that there are, from 2^31 on), but the next lower logit is 128 less, so that
// a term is 2^((x - m) log2(e)), 1 or as good as 0, and a sum is forgotten at a new reference.
//   The best tokens: the width-th highest of the lanes' maxima is a bound that no lane with a lower maximum reaches, which leaves `width`
// lanes (more where there are ties); the tiles of theirs whose maximum reaches it, too, are read again and compared.  (Looked for in every tile, as the row goes by, they cost
// twice the instructions of all the rest: 96 x 5 rows of 99991 65 us, so 41; all pieces of those lanes, 41, their best tiles' only, 38.)
struct Part {
  uint32_t best = 0;            // lane i: the i-th best: the logit's order above, the place from behind below: no two are equal
  double sum = 0.0, ref = 0.0;  // sum of e^x = sum e^ref; ref the same in all lanes
};
constexpr uint32_t WAITING = 768;      // a turn adds 512 at most
constexpr uint32_t TOPS = 4;            // tiles' maxima at a time
struct PartSpace { uint32_t waiting[WAITING], pieces[32 + TOPS * 64 + 32]; };
template <class Counts>
__device__ __forceinline__ Part part_of(const bf16_t* x, uint32_t v0, uint32_t v1, uint32_t width, PartSpace& space, uint16_t* tops, Counts&& counts) {
  uint32_t* const waiting = space.waiting;
  const uint32_t lane = threadIdx.x & 63u;
  // whole 16-byte pieces as they lie in memory; the up to seven logits before them and those behind them one a lane (0 .. 6, 8 .. 14)
  const uint32_t before = min((uint32_t)(-((uintptr_t)(x + v0) / 2u)) & 7u, v1 - v0), pieces = (v1 - v0 - before) / 8u, behind = (v1 - v0 - before) % 8u;
  const bf16_t* const whole = x + v0 + before;
  auto piece = [&](uint32_t i) { return *reinterpret_cast<const uint4*>(whole + (uint64_t)i * 8u); };
  struct Tile { uint32_t d[LANE / 2]; };
  // (loaded without a branch around it; what lies beyond is the last piece again and is taken out when its turn comes)
  auto load = [&](uint32_t i) {
    Tile t;
#pragma unroll
    for (uint32_t u = 0; u < LANE / 8; ++u) {
      const uint4 q = piece(min(i * (TILE / 8u) + u * 64u + lane, pieces - 1u));
      t.d[u * 4] = q.x; t.d[u * 4 + 1] = q.y; t.d[u * 4 + 2] = q.z; t.d[u * 4 + 3] = q.w;
    }
    return t;
  };
  constexpr uint32_t NONE = 0xff80ff80u;
  const uint32_t n_tiles = (pieces + TILE / 8u - 1u) / (TILE / 8u);
  const uint32_t edge_at = lane < 8u ? lane : v1 - v0 - behind + (lane - 8u);
  uint32_t edge = NONE;
  if (lane < before || (lane >= 8u && lane < 8u + behind)) edge = 0xff800000u | x[v0 + edge_at];
  Tile next = {};
  if (n_tiles) next = load(0);
  Part p;
  if (!counts()) return p;
  float m = 0.0f, c = 0.0f, lane_top = -INFINITY;     // m: what c stands for
  bool some = false, large = false;
  auto any = [](bool b) { return __ballot(b) != 0; };
  // Dwords d[0 .. n - 1] of two logits each.
  auto add = [&](const uint32_t* d, auto n) {
    constexpr uint32_t N = decltype(n)::value;
    float top = -INFINITY;
#pragma unroll
    for (uint32_t u = 0; u < N; ++u) top = fmaxf(fmaxf(top, low_half(d[u])), high_half(d[u]));
    auto refer_to = [&](float tile_top) {          // a new reference, where these logits ask for one
      if (!any(tile_top > -INFINITY && (!some || (tile_top - m) * LOG2E > HIGHEST))) return;
      float m2 = some ? fmaxf(m, tile_top) : tile_top;
      m2 = unordered(wave_top(ordered(m2)));
      const float c2 = m2 * LOG2E;
      const bool large2 = !(fabsf(m2) < LARGE);
      p.sum = some && !large && !large2 ? p.sum * exp2((double)c - (double)c2) : 0.0;
      m = m2; c = c2; some = true;
      large = large2;
    };
    bool odd = any(top == INFINITY);
    if (!odd) { refer_to(top); odd = large; }
    if (!odd) {
      float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < N; ++u) {
        s0 += __builtin_amdgcn_exp2f(__builtin_fmaf(low_half(d[u]), LOG2E, -c));
        s1 += __builtin_amdgcn_exp2f(__builtin_fmaf(high_half(d[u]), LOG2E, -c));
      }
      const float s = s0 + s1;
      odd = any(!(s < INFINITY));
      if (!odd) p.sum += (double)s;
    }
    if (odd) {
      top = -INFINITY;
#pragma unroll
      for (uint32_t u = 0; u < 2 * N; ++u) {
        const uint32_t o = order_of(d[u / 2] >> 16 * (u & 1) & 0xffffu);
        top = fmaxf(top, o ? value_of(o) : -INFINITY);
      }
      refer_to(top);
      float s = 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < 2 * N; ++u) {
        const uint32_t o = order_of(d[u / 2] >> 16 * (u & 1) & 0xffffu);
        const float v = value_of(o);
        s += o ? __builtin_amdgcn_exp2f(large ? (v - m) * LOG2E : __builtin_fmaf(v, LOG2E, -c)) : 0.0f;
      }
      p.sum += (double)s;
    }
    lane_top = fmaxf(lane_top, top);
    return top;
  };
#pragma unroll 1
  for (uint32_t i = 0; i < n_tiles; ++i) {
    Tile t = next;
    next = load(min(i + 1, n_tiles - 1));
    if (i == n_tiles - 1) {
#pragma unroll
      for (uint32_t u = 0; u < LANE / 2; ++u) t.d[u] = i * (TILE / 8u) + u / 4 * 64u + lane < pieces ? t.d[u] : NONE;
    }
    tops[i * 64u + lane] = (uint16_t)(__float_as_uint(add(t.d, std::integral_constant<uint32_t, LANE / 2>{})) >> 16);
  }
  if (before + behind) add(&edge, std::integral_constant<uint32_t, 1>{});
  p.ref = large ? (double)m : (double)m + ((double)c - (double)m * (double)LOG2E) * LN2;        // 2^(x LOG2E - c) stands for e^(x - m) 2^(m LOG2E - c)
  p.sum = wave_total(p.sum);

  // ---- the best
  float bound = -INFINITY;
  {
    uint32_t tops = lane_top > -INFINITY ? order_of(__float_as_uint(lane_top) >> 16) << 6 | lane : 0u, got = 1;
#pragma unroll 1
    for (uint32_t r = 0; r < width && got; ++r) {
      got = wave_top(tops);
      tops = tops == got ? 0u : tops;
    }
    if (got) bound = value_of(got >> 6);
  }
  uint32_t n_waiting = 0;
  auto sort_out = [&]() {
#pragma unroll 1
    for (uint32_t first = 0; first < n_waiting; first += 128u) {
      uint32_t k0 = first + lane < n_waiting ? waiting[first + lane] : 0u, k1 = first + lane + 64u < n_waiting ? waiting[first + lane + 64u] : 0u;
      uint32_t k2 = p.best, top = max(max(k0, k1), k2), best = 0, got = 1;
#pragma unroll 1
      for (uint32_t r = 0; r < width && got; ++r) {
        got = wave_top(top);
        best = lane == r ? got : best;
        k0 = k0 == got ? 0u : k0; k1 = k1 == got ? 0u : k1; k2 = k2 == got ? 0u : k2;
        top = max(max(k0, k1), k2);
      }
      p.best = best;
    }
    n_waiting = 0;
  };
  auto wait = [&](uint32_t bits, uint32_t place) {           // of every lane one logit, or none
    const uint32_t o = __uint_as_float(bits << 16) >= bound ? order_of(bits) : 0u;
    const uint64_t who = __ballot(o != 0u);
    if (!who) return;
    if (o) waiting[n_waiting + (uint32_t)__popcll(who & ((1ull << lane) - 1ull))] = o << 16 | (MAX_SPAN - 1u - place);
    n_waiting += (uint32_t)__popcll(who);
  };
  if (before + behind) wait(edge & 0xffffu, edge_at);
  // a lane's two pieces of every tile in which it reaches the bound are read again, one a lane
  const uint64_t lower = (1ull << lane) - 1ull;
  uint32_t n_found = 0;
#pragma unroll 1
  for (uint32_t first = 0; first < n_tiles; first += TOPS) {
    float top[TOPS];
#pragma unroll
    for (uint32_t u = 0; u < TOPS; ++u) {
      top[u] = __uint_as_float((uint32_t)tops[min(first + u, n_tiles - 1u) * 64u + lane] << 16);
      if (first + u >= n_tiles || !(top[u] >= bound)) top[u] = -INFINITY;
    }
#pragma unroll
    for (uint32_t u = 0; u < TOPS; ++u) {
      const uint64_t found = __ballot(top[u] > -INFINITY);
      if (!found) continue;
      const uint32_t at = (first + u) * 128u + lane;
      if (found >> lane & 1u) space.pieces[n_found / 2u + (uint32_t)__popcll(found & lower)] = at | (at + 64u) << 16;
      n_found += 2u * (uint32_t)__popcll(found);
    }
    const bool last = first + TOPS >= n_tiles;
    if (!n_found || (n_found < 64u && !last)) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    uint32_t done = 0;
    for (; done < n_found && (last || n_found - done >= 64u); done += 64u) {
      const uint32_t k = min(done + lane, n_found - 1u), at = space.pieces[k / 2u] >> 16u * (k & 1u) & 0xffffu;
      const bool there = done + lane < n_found && at < pieces;
      const uint4 q = piece(min(at, pieces - 1u));
      const uint32_t d[4] = {q.x, q.y, q.z, q.w};
      if (n_waiting > WAITING - 512u) sort_out();
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) wait(there ? d[u / 2] >> 16 * (u & 1) & 0xffffu : 0xff80u, before + at * 8u + u);
    }
    if (last) break;
    const uint32_t left = n_found - done, x = space.pieces[done / 2u + (lane & 31u)];       // less than a wavefront's: for the next turn
    if (2u * lane < left) space.pieces[lane] = x;
    n_found = left;
  }
  sort_out();
  return p;
}

// A candidate: the higher key first, then the lower place (beam and token).  order: the key's bits as a number that orders like it, 0 none.
struct Candidate {
  uint64_t order = 0;
  uint32_t place = ~0u;
  __device__ __forceinline__ bool before(const Candidate& o) const { return order > o.order || (order == o.order && place < o.place); }
};
__device__ __forceinline__ uint64_t ordered(double key) {
  const uint64_t b = __builtin_bit_cast(uint64_t, key + 0.0);          // 0 for -0
  return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ Candidate wave_first(const Candidate& c) {
  Candidate r;
  const uint32_t high = (uint32_t)(c.order >> 32), low = (uint32_t)c.order, top = wave_top(high);
  const uint64_t who = __ballot(high == top);
  if (__popcll(who) == 1) {                                             // most often: the rest need not be compared
    const int lane = (int)__builtin_ctzll(who);
    r.order = (uint64_t)top << 32 | (uint32_t)__builtin_amdgcn_readlane((int)low, lane);
    r.place = (uint32_t)__builtin_amdgcn_readlane((int)c.place, lane);
    return r;
  }
  const uint32_t next = wave_top(high == top ? low : 0u);
  r.order = (uint64_t)top << 32 | next;
  r.place = ~wave_top(high == top && low == next ? ~c.place : 0u);
  return r;
}

// 96 x 5 rows of 99991 (88 MB, 14.5 us of reading): 35.6 us; exponentials beside the loads, then the hand-over to a prompt's last workgroup, its lists,
// rounds and states, some 10 us of which the last prompts' show.  1 x 4 rows of 32000: 12.6 us, all latency: a part 4, the hand-over 1.7, lists and
// sums 2.3, rounds 2.5, states 1.4.
// One launch.  Every wavefront takes a part of a row; the last workgroup of a prompt to be done finds its beams among the parts' best, each list of
// them in order; the last prompt's packs the tokens.
constexpr uint32_t STAGED = 8192;                                        // best tokens of all parts that fit the LDS
constexpr uint32_t HELD = 16, EARLY = 8;
__global__ __launch_bounds__(THREADS) void beam_select_kernel(BeamArgs a) {
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t W = a.width, lists = W * a.parts, group = blockIdx.x / a.wgs, r0 = group * W;
  __shared__ double lse[BEAM_MAX_WIDTH], score[BEAM_MAX_WIDTH], factor[BEAM_MAX_WIDTH];        // factor: what a beam's totals are divided by
  __shared__ int32_t count[BEAM_MAX_WIDTH], parent[BEAM_MAX_WIDTH], token[BEAM_MAX_WIDTH];
  __shared__ PartSpace space[WAVES];
  __shared__ uint32_t kind[BEAM_MAX_WIDTH];                                                     // 0: none, 1: goes on, 2: has ended
  extern __shared__ uint32_t staged[];    // a part's tiles' maxima; then the parts' best tokens and a cursor for every list but a thread's first
  float old_score = -INFINITY;
  int32_t old_count = 0, old_ended = 0;
  if (tid < W) { old_score = a.scores[r0 + tid]; old_count = a.counts[r0 + tid]; old_ended = a.ended[r0 + tid]; }
  {
    const uint32_t w = (blockIdx.x % a.wgs) * WAVES + wave, b = w / a.parts, part = w % a.parts, row = r0 + b;
    if (w < lists) {
      const uint32_t v0 = part * a.span;
      // (a beam that is none, or has ended: nobody asks for what is left here)
      const Part p = part_of(a.logits + (uint64_t)row * a.ld, v0, min(v0 + a.span, a.vocab), W, space[wave], (uint16_t*)staged + (uint64_t)wave * a.tiles * 64u, [&] { return !a.ended[row] && a.scores[row] > -INFINITY; });
      const uint64_t list = (uint64_t)group * lists + w;
      if (lane < W) share_out(a.best + list * W + lane, p.best);
      if (lane == 0) { share_out(a.sums + 2 * list, p.sum); share_out(a.sums + 2 * list + 1, p.ref); }
    }
  }
  if (tid < W) {
    const int32_t n = max(0, old_count);
    const uint32_t k = !(old_score > -INFINITY) ? 0u : old_ended ? 2u : 1u;
    kind[tid] = k; score[tid] = (double)old_score; count[tid] = n;
  }
  __shared__ uint32_t flag;
  if (!last_of(a.counters + 1 + group, a.wgs, &flag)) return;

  __shared__ uint64_t found_order[WAVES][BEAM_MAX_WIDTH];
  __shared__ uint32_t found_place[WAVES][BEAM_MAX_WIDTH], found_logit[WAVES][BEAM_MAX_WIDTH];
  const bool stage = lists * W <= STAGED;
  uint8_t* const cursor = (uint8_t*)(staged + (stage ? lists * W : 0u));
  const uint32_t* const best = a.best + (uint64_t)group * lists * W;
  // the histories' old columns are on their way from here on, where they are few
  uint32_t longest_old = 0;
  for (uint32_t b = 0; b < W; ++b)
    if (kind[b]) longest_old = max(longest_old, min((uint32_t)count[b], a.max_history));
  const bool short_ones = longest_old <= THREADS * EARLY / W;
  int32_t* const histories = (int32_t*)space;                    // the parts are done
  static_assert(sizeof(space) >= THREADS * EARLY * 4);
  int32_t early[EARLY];
#pragma unroll
  for (uint32_t u = 0; u < EARLY; ++u) {
    const uint32_t e = u * THREADS + tid;
    if (short_ones && e < longest_old * W) early[u] = a.history[(uint64_t)(r0 + e / longest_old) * a.max_history + e % longest_old];
  }
  for (uint32_t b = wave; b < W; b += WAVES) {
    double sum = 0.0, ref = -INFINITY;
    const uint32_t k = kind[b];
    if (k == 1u && lane < a.parts) {
      const double* const from = a.sums + 2 * ((uint64_t)group * lists + b * a.parts + lane);
      sum = shared_in(from);
      ref = shared_in(from + 1);
      if (!(sum > 0.0)) ref = -INFINITY;
    }
    if (stage && b == wave)
      for (uint32_t i = tid; i < lists * W; i += THREADS) staged[i] = shared_in(best + i);
    if (lane == 0) factor[b] = a.penalty == 0.0 ? 1.0 : pow((double)max(1, k == 1u && count[b] < INT32_MAX ? count[b] + 1 : count[b]), a.penalty);
    if (k != 1u) continue;
    const double top = (double)unordered(wave_top(ordered((float)ref)));           // the highest, or next to it
    const double all = wave_total(sum > 0.0 ? sum * exp(ref - top) : 0.0);
    if (lane == 0) lse[b] = log(all) + top;
  }
  if (stage && wave >= W)                       // (a wavefront without a beam)
    for (uint32_t i = tid; i < lists * W; i += THREADS) staged[i] = shared_in(best + i);
#pragma unroll
  for (uint32_t u = 0; u < EARLY; ++u)
    if (short_ones && u * THREADS + tid < longest_old * W) histories[u * THREADS + tid] = early[u];
  __syncthreads();
  auto total_of = [&](uint32_t b, float x) { return kind[b] == 2u ? score[b] : ((double)x - lse[b]) + score[b]; };
  // a list: a part of beam b; its at-th best token, from place v0 on
  auto candidate = [&](uint32_t list, uint32_t b, uint32_t part, uint32_t at, uint32_t* key_out) {
    Candidate c;
    const uint32_t k = kind[b];
    uint32_t key = 0;
    if (k == 2u) {
      if (part == 0 && at == 0) { c.order = ordered(score[b] / factor[b]); c.place = b * a.vocab + (uint32_t)max(a.end_token, 0); }
    } else if (k == 1u && at < W) {
      key = stage ? staged[list * W + at] : shared_in(best + list * W + at);
      if (key) {
        const double t = ((double)value_of(key >> 16) - lse[b]) + score[b];
        c.order = ordered(a.penalty == 0.0 ? t : t / factor[b]);
        c.place = b * a.vocab + part * a.span + (MAX_SPAN - 1u - (key & 0xffffu));
      }
    }
    *key_out = key;
    return c;
  };
  // every wavefront the best of its lists, then the first one the best of theirs; where one wavefront has all lists it has them at once
  const uint32_t have = min(WAVES, (lists + 63) / 64);
  if (wave < have) {
    // a thread's first list, which mostly is its only one: what its candidates are made of in registers
    const uint32_t own_b = min(tid / a.parts, W - 1u), own_part = tid % a.parts, own_kind = tid < lists ? kind[own_b] : 0u;
    const double own_lse = lse[own_b], own_score = score[own_b], own_factor = factor[own_b];
    uint32_t own_at = 0, own_key = 0, key = 0, from = tid;
    Candidate own, mine;
    auto own_candidate = [&]() {
      own = Candidate{};
      if (own_kind != 1u) {
        if (own_kind == 2u) own = candidate(tid, own_b, own_part, own_at, &own_key);
        return;
      }
      own_key = own_at < W ? stage ? staged[tid * W + own_at] : shared_in(best + tid * W + own_at) : 0u;
      if (!own_key) return;
      const double t = ((double)value_of(own_key >> 16) - own_lse) + own_score;
      own.order = ordered(a.penalty == 0.0 ? t : t / own_factor);
      own.place = own_b * a.vocab + own_part * a.span + (MAX_SPAN - 1u - (own_key & 0xffffu));
    };
    own_candidate();
    mine = own; key = own_key;
    for (uint32_t l = tid + THREADS; l < lists; l += THREADS) {
      uint32_t k;
      cursor[l] = 0;
      const Candidate c = candidate(l, l / a.parts, l % a.parts, 0, &k);
      if (c.before(mine)) { mine = c; key = k; from = l; }
    }
    for (uint32_t r = 0; r < W; ++r) {
      const Candidate c = wave_first(mine);
      if (!c.order) {
        for (uint32_t x = r + lane; x < W; x += 64) found_order[wave][x] = 0;
        break;
      }
      if (mine.place == c.place && mine.order) {
        found_order[wave][r] = c.order; found_place[wave][r] = c.place; found_logit[wave][r] = key;
        if (from == tid) { ++own_at; own_candidate(); }
        else ++cursor[from];
        mine = own; key = own_key; from = tid;
        for (uint32_t l = tid + THREADS; l < lists; l += THREADS) {
          uint32_t k;
          const Candidate d = candidate(l, l / a.parts, l % a.parts, cursor[l], &k);
          if (d.before(mine)) { mine = d; key = k; from = l; }
        }
      }
    }
  }
  __syncthreads();
  uint64_t order = 0;
  uint32_t place = 0, key = 0;
  if (wave == 0) {
    if (have == 1) {
      if (lane < W) { order = found_order[0][lane]; place = found_place[0][lane]; key = found_logit[0][lane]; }
    } else {
      uint32_t at = 0;
      Candidate mine;
      if (lane < have) { mine.order = found_order[lane][0]; mine.place = found_place[lane][0]; }
      for (uint32_t r = 0; r < W; ++r) {
        const Candidate c = wave_first(mine);
        if (!c.order) break;
        const bool won = mine.place == c.place && mine.order;
        const uint32_t k = won ? found_logit[lane][at] : 0u, winner = (uint32_t)__builtin_ctzll(__ballot(won));
        if (lane == r) { order = c.order; place = c.place; }
        const uint32_t of_winner = (uint32_t)__builtin_amdgcn_readlane((int)k, (int)winner);
        if (lane == r) key = of_winner;
        if (won) {
          ++at;
          mine = Candidate{};
          if (at < W) { mine.order = found_order[lane][at]; mine.place = found_place[lane][at]; }
        }
      }
    }
    if (lane < W) {
      parent[lane] = order ? (int32_t)(place / a.vocab) : -1;
      token[lane] = order ? (int32_t)(place % a.vocab) : -1;
    }
  }
  __syncthreads();
  // ---- states (stored behind the barrier: it would wait for them)
  if (tid < W) {
    const bool found = order != 0;
    const uint32_t r = r0 + tid, b = found ? (uint32_t)parent[tid] : 0u;
    const int32_t v = token[tid];
    float s = -INFINITY;
    int32_t n = 0, ended = 1;
    if (found) {
      const bool was = kind[b] == 2u;
      s = (float)total_of(b, value_of(key >> 16));
      n = was || count[b] == INT32_MAX ? count[b] : count[b] + 1;
      ended = was || v == a.end_token;
    }
    a.scores[r] = s;
    a.counts[r] = n;
    a.ended[r] = ended;
    a.parents[r] = found ? (int32_t)(r0 + b) : -1;
    share_out((uint32_t*)a.chosen + r, (uint32_t)v);
    share_out((uint32_t*)a.added + r, !ended);
    if (a.n_rows == W) {                         // a single prompt: its tokens are all there are
      const uint64_t on = __ballot(!ended), lower = (1ull << lane) - 1ull, here = __ballot(true);
      const uint32_t ahead = (uint32_t)__popcll(on & lower), behind = (uint32_t)__popcll(on) + (uint32_t)__popcll(here & ~on & lower);
      a.tokens[ended ? behind : ahead] = ended ? 0 : v;
    }
  }
  // histories, some columns of all rows at a time: read, then written
  uint32_t longest = 0;
  for (uint32_t b = 0; b < W; ++b)
    if (parent[b] >= 0) longest = max(longest, min((uint32_t)count[parent[b]] + 1u, a.max_history));
  auto each = [&](uint32_t c0, uint32_t n, auto&& f) {
#pragma unroll
    for (uint32_t u = 0; u < HELD; ++u) {
      const uint32_t e = u * THREADS + tid;
      if (e >= n * W) break;
      const uint32_t i = e / n, c = c0 + e % n;
      if (parent[i] < 0) continue;
      const uint32_t b = (uint32_t)parent[i], end = (uint32_t)count[b];
      if (c < end || (c == end && kind[b] == 1u)) f(u, i, b, c, end);
    }
  };
  if (short_ones && longest <= THREADS * HELD / W) {
    each(0, longest, [&](uint32_t, uint32_t i, uint32_t b, uint32_t c, uint32_t end) {
      if (c < end && b == i) return;
      a.history[(uint64_t)(r0 + i) * a.max_history + c] = c < end ? histories[b * longest_old + c] : token[i];
    });
  } else {
    const uint32_t columns = THREADS * HELD / W;
    for (uint32_t c0 = 0; c0 < longest; c0 += columns) {
      const uint32_t n = min(columns, longest - c0);
      int32_t held[HELD];
      each(c0, n, [&](uint32_t u, uint32_t i, uint32_t b, uint32_t c, uint32_t end) { held[u] = c < end ? a.history[(uint64_t)(r0 + b) * a.max_history + c] : token[i]; });
      __syncthreads();
      each(c0, n, [&](uint32_t u, uint32_t i, uint32_t, uint32_t c, uint32_t) { a.history[(uint64_t)(r0 + i) * a.max_history + c] = held[u]; });
      __syncthreads();
    }
  }
  // ---- the tokens of the beams that go on, one behind the other
  if (a.n_rows == W || !last_of(a.counters, a.n_rows / W, &flag)) return;
  __shared__ uint32_t red[WAVES];
  const uint32_t per = (a.n_rows + THREADS - 1) / THREADS, first = min(tid * per, a.n_rows), end = min(first + per, a.n_rows);
  uint32_t on = 0, all = 0;
#pragma unroll 4
  for (uint32_t j = first; j < end; ++j) on += shared_in((uint32_t*)a.added + j);
  const uint32_t upto = lane_scan(on);
  uint32_t at = upto - on;
  if (lane == 63u) red[wave] = upto;
  __syncthreads();
  for (uint32_t w = 0; w < WAVES; ++w) {
    if (w < wave) at += red[w];
    all += red[w];
  }
  for (uint32_t j = first; j < end; ++j) {
    if (shared_in((uint32_t*)a.added + j)) a.tokens[at++] = (int32_t)shared_in((uint32_t*)a.chosen + j);
    if (j >= all) a.tokens[j] = 0;
  }
}

// Parts of a row: enough wavefronts for the chip (rows of 99991, five a prompt, with 1536 / 2048 / 3072 / 4096 wavefronts: 480 rows 38.5 / 35.6 / 36.3 / 37.3 us,
// 80 rows 25.5 / 26.4 / 28.5 / 31.9), two tiles at least for each (4 rows of 32000 in 32 parts of one: 1 us more, for the lists that there are then).
constexpr uint32_t WANTED_WAVES = 2048;
void cut(uint32_t n_rows, uint32_t vocab, uint32_t* parts, uint32_t* span) {
  uint32_t p = std::min((vocab + 2 * TILE - 1) / (2 * TILE), std::max(1u, WANTED_WAVES / n_rows));
  p = std::min(std::max(p, (vocab + MAX_SPAN - 1) / MAX_SPAN), MAX_PARTS);
  *span = std::min(((vocab + p - 1) / p + 7) / 8 * 8, MAX_SPAN);
  *parts = (vocab + *span - 1) / *span;
}
uint64_t up16(uint64_t bytes) { return (bytes + 15) & ~15ull; }

}  // namespace

uint64_t beam_select_scratch(uint32_t n_rows, uint32_t width, uint32_t vocab) {
  uint32_t parts, span;
  cut(n_rows, vocab, &parts, &span);
  return BEAM_COUNTERS * 4 + 16ull * n_rows * parts + up16(4ull * n_rows * parts * width);
}

hipError_t launch_beam_select(BeamArgs a, void* scratch, hipStream_t st) {
  cut(a.n_rows, a.vocab, &a.parts, &a.span);
  a.counters = (uint32_t*)scratch;
  a.sums = (double*)((char*)scratch + BEAM_COUNTERS * 4);
  a.best = (uint32_t*)((char*)a.sums + 16ull * a.n_rows * a.parts);
  a.wgs = (a.width * a.parts + WAVES - 1) / WAVES;
  a.tiles = (a.span / 8 + TILE / 8 - 1) / (TILE / 8);
  const uint32_t lists = a.width * a.parts, lds = std::max(WAVES * a.tiles * 128, (lists * a.width <= STAGED ? lists * a.width * 4 : 0) + lists);
  beam_select_kernel<<<a.n_rows / a.width * a.wgs, THREADS, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace qzo
