// Attention of the newest tokens of sequences over a paged cache of keys and values.
//
// out = sum_k p_k v_k / sum_k p_k, p_k = 2^(s_k - m), s_k = q . k scale log2(e), m a running maximum: one pass over the keys.
// A key head's keys and values are read once for all queries that share it: 16 of them (heads of the group, token by token)
// are the columns of one matrix tile, so that a single query costs what sixteen do, and the memory is what counts.
//
//   S[key][col]  = K Q^T     v_mfma_f32_16x16x32_bf16, 16 keys a tile, K's rows straight from memory as the first operand
//   O[dim][col] += V^T P^T   32 keys an instruction
// The second product takes S's own registers: a lane holds column lane % 16 and keys 4 (lane / 16) + 0..3 of two tiles, which
// are eight of the 32 values of k that its place of the operand is to hold, if V's rows are dealt out the same way.  V comes
// in rows too (16 lanes read a row, VW = DH / 16 features each, a lane the eight rows of its keys) and is transposed in
// registers, eight 16-bit columns at a time, with one v_perm_b32 per pair of keys.  No LDS, no exchange between lanes but for
// the maximum, and that only when it has grown by a factor of 2^8: until then the sums carry the larger terms.
// All of a column's state (maximum, sum, its 4 VW accumulators) is in the lanes that hold the column.
//
// What bounds it: memory.  A step of a wavefront loads its next 32 keys (16 KB at heads of 128, bf16) before it works on the
// ones it has; eight wavefronts on a compute unit keep 128 KB on the way.
#include <algorithm>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// How the work is dealt out.  A group is a column tile of one sequence and key head; it has units of 128 keys, and SETUP more
// that stand for what a group costs apart from its keys.  All groups' units are counted through, and workgroup b takes units
// b per .. (b + 1) per - 1: every workgroup the same share, whatever the lengths.  A group that lies in one workgroup's share
// is written by it; otherwise each leaves (maximum, sum, accumulators) in the scratch, its first group's in place 2 b, a later
// one's (only the last can go on) in 2 b + 1, and who finds the group's counter at its last piece adds them up, in order.  The
// counter (that of the workgroup of the group's first piece) goes back to zero for the next call.
constexpr uint32_t UNIT = 128, COLS = 16, WAVES = 4, MAX_WGS = 512;
constexpr uint32_t SETUP = 2, MIN_SHARE = 6;

struct SeqWork { uint32_t row0, rows, len, units, tiles; };

__device__ __forceinline__ SeqWork seq_work(const PagedArgs& a, uint32_t i) {
  SeqWork w;
  w.row0 = i; w.rows = i < a.n_rows ? 1u : 0u;
  if (a.starts) {
    const int32_t s0 = min(max(a.starts[i], 0), (int32_t)a.n_rows), s1 = min(max(a.starts[i + 1], s0), (int32_t)a.n_rows);
    w.row0 = (uint32_t)s0; w.rows = (uint32_t)(s1 - s0);
  }
  w.len = (uint32_t)min(max(a.lengths[i], 0), (int32_t)(a.max_blocks << a.block_shift));
  w.units = max(1u, (w.len + UNIT - 1) / UNIT);
  w.tiles = (uint32_t)(((uint64_t)w.rows * a.group + COLS - 1) / COLS);
  return w;
}

// What all lanes agree on, in a scalar register.
__device__ __forceinline__ uint32_t scalar(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ uint64_t scalar64(uint64_t x) { return (uint64_t)scalar((uint32_t)(x >> 32)) << 32 | scalar((uint32_t)x); }

// Two floats for another workgroup, on any XCD: stored through the L2 and loaded past it (agent scope), so that no L2 has to be
// written back or invalidated as a whole, which a fence of that scope does (64 ragged sequences: 366 us with fences).  A
// wavefront's stores have arrived when its count of outstanding ones is zero; it raises the group's counter after that.
__device__ __forceinline__ void share_out(float* p, float x, float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void shared_out() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ float2 shared_in(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Four accumulators of a column, of several pieces of its keys.
struct Joined {
  float m = -INFINITY, l = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  __device__ __forceinline__ void add(float m1, float l1, const f32x4& o1) {
    if (m1 == -INFINITY && l1 == 0.0f) return;           // saw nothing (a NaN goes on)
    const float top = fmaxf(m, m1), f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top), f1 = __builtin_amdgcn_exp2f(m1 - top);
    l = l * f + l1 * f1;
    o = o * f + o1 * f1;
    m = top;
  }
};

template <class T>
__device__ __forceinline__ T block_scan(T v, T* total, T* red) {     // exclusive, 256 threads
  T s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(s, o, 64);
    if ((threadIdx.x & 63u) >= (uint32_t)o) s += u;
  }
  __syncthreads();
  if ((threadIdx.x & 63u) == 63u) red[threadIdx.x >> 6] = s;
  __syncthreads();
  T before = 0, all = 0;
  for (uint32_t w = 0; w < WAVES; ++w) {
    if (w < (threadIdx.x >> 6)) before += red[w];
    all += red[w];
  }
  *total = all;
  return before + s - v;
}

__device__ __forceinline__ uint32_t two_bf16(uint32_t raw, bool high) {      // two e4m3 bytes of a dword as two bf16
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  const bf2 v = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw, 1.0f, false);
  return __builtin_bit_cast(uint32_t, v);
}

// Whether a dword of values holds a NaN or an infinity (e4m3 has no infinities).
template <bool E4M3>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
  if (E4M3) return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// KP: pairs of key tiles a step.
template <int DH, bool E4M3, int KP>
struct PagedStep {
  static constexpr int KL = E4M3 ? DH / 64 : DH / 32;      // 16-byte loads a key tile takes
  static constexpr int VD = E4M3 ? DH / 64 : DH / 32;      // dwords of a row of V that a lane holds
  u32x4v k[KP][2][KL];
  uint32_t v[KP][8][VD];
};

template <int DH, bool E4M3, int KP>
__global__ __launch_bounds__(256, 2) void paged_attention_kernel(PagedArgs a, uint32_t* counters, float* parts, uint32_t part_cols) {
  constexpr int KS = DH / 32, VW = DH / 16, ES = E4M3 ? 1 : 2;
  constexpr uint32_t STEP = 32 * KP, ROUND = STEP * WAVES;
  typedef PagedStep<DH, E4M3, KP> Step;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  float* const sum_acc = (float*)lds;                                   // [WAVES][COLS][DH + 4]
  float* const sum_m = sum_acc + WAVES * COLS * (DH + 4);               // [WAVES][COLS]
  float* const sum_l = sum_m + WAVES * COLS;
  uint64_t* const red = (uint64_t*)(sum_l + WAVES * COLS);              // [WAVES]
  uint64_t* const first_unit = red + WAVES;                             // [n_seq], more than 64 sequences only
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = scalar(tid >> 6);
  const uint32_t col = lane & 15u, g = lane >> 4;

  // ---- the sequences' units: up to 64 sequences in the lanes of every wavefront, more in the LDS
  const bool few = a.n_seq <= 64;
  uint64_t total, mine = 0;
  SeqWork lane_work = {0, 0, 0, 1, 0};
  if (few) {
    uint64_t n = 0;
    if (lane < a.n_seq) {
      lane_work = seq_work(a, lane);
      n = (uint64_t)(lane_work.units + SETUP) * lane_work.tiles * a.kv_heads;
    }
    uint64_t s = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t u = __shfl_up(s, o, 64);
      if (lane >= (uint32_t)o) s += u;
    }
    total = __shfl(s, 63, 64);
    mine = s - n;
  } else {
    const uint32_t per = (a.n_seq + 255) / 256, s_first = min(tid * per, a.n_seq), s_last = min(s_first + per, a.n_seq);
    uint64_t n = 0;
    for (uint32_t i = s_first; i < s_last; ++i) {
      const SeqWork w = seq_work(a, i);
      first_unit[i] = n;
      n += (uint64_t)(w.units + SETUP) * w.tiles * a.kv_heads;
    }
    const uint64_t before = block_scan(n, &total, red);
    for (uint32_t i = s_first; i < s_last; ++i) first_unit[i] += before;
    __syncthreads();
  }
  total = scalar64(total);
  const uint64_t share = max((uint64_t)MIN_SHARE, (total + gridDim.x - 1) / gridDim.x);
  // neighbours (the column tiles of the same keys) on one XCD; the grid is a multiple of 8
  const uint32_t wg = (blockIdx.x & 7u) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  const uint64_t begin = share * wg, end = min(begin + share, total);

  for (uint64_t unit = begin; unit < end;) {
    uint32_t seq;
    uint64_t seq_first;
    SeqWork w;
    if (few) {
      // prefixes ascend and begin at 0: the last one not above is the sequence that has the unit
      seq = scalar((uint32_t)__popcll(__ballot(lane < a.n_seq && mine <= unit)) - 1u);
      seq_first = (uint64_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, (int)seq) & 0xffffffffu;
      seq_first |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), (int)seq) << 32;
      auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)seq); };
      w = {of(lane_work.row0), of(lane_work.rows), of(lane_work.len), of(lane_work.units), of(lane_work.tiles)};
    } else {
      uint32_t lo = 0, hi = a.n_seq;
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first_unit[mid] <= unit) lo = mid; else hi = mid;
      }
      seq = scalar(lo);
      seq_first = scalar64(first_unit[seq]);
      w = seq_work(a, seq);
      w = {scalar(w.row0), scalar(w.rows), scalar(w.len), scalar(w.units), scalar(w.tiles)};
    }
    const uint32_t span = w.units + SETUP;
    const uint64_t r = unit - seq_first;
    const uint32_t group = scalar((r >> 32) ? (uint32_t)(r / span) : (uint32_t)r / span);
    const uint32_t tile = scalar(group % w.tiles), kh = scalar(group / w.tiles);
    const uint32_t at = scalar((uint32_t)(r - (uint64_t)group * span));                     // within the group, SETUP first
    const uint32_t n_units = scalar((uint32_t)min((uint64_t)(span - at), end - unit));
    const uint64_t group_first = unit - at + SETUP, group_last = unit - at + span - 1;
    const bool at_begin = unit == begin;
    unit += n_units;
    if (at + n_units <= SETUP) continue;
    const uint32_t u_first = max(at, SETUP) - SETUP, u_end = at + n_units - SETUP;
    const uint32_t wg_first = group_first >= begin ? wg : wg - scalar((uint32_t)((begin - group_first + share - 1) / share));
    const uint32_t wg_last = group_last < end ? wg : wg + scalar((uint32_t)((group_last - end) / share)) + 1u, pieces = wg_last - wg_first + 1u;

    // ---- this tile's columns
    const uint32_t flat = tile * COLS + col, token = flat / a.group, head = kh * a.group + flat % a.group;
    const uint32_t n_cols = min(COLS, w.rows * a.group - tile * COLS);
    const bool live = col < n_cols;
    const uint64_t row = w.row0 + (live ? token : 0u);
    const int32_t sees = live ? (int32_t)(w.len + token + 1u - w.rows) : 0;                  // positions that the column sees
    const int32_t least = (int32_t)(w.len + tile * COLS / a.group + 1u - w.rows);             // the first column's, the fewest
    const int32_t most = (int32_t)(w.len + (tile * COLS + n_cols - 1) / a.group + 1u - w.rows);
    const int32_t k_first = (int32_t)(u_first * UNIT), k_end = (int32_t)min((int64_t)most, (int64_t)u_end * UNIT);

    bf16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      // e4m3: a 16-byte load of K is two operands
      const uint32_t d = E4M3 ? (uint32_t)(s / 2) * 64u + g * 16u + (uint32_t)(s & 1) * 8u : (uint32_t)s * 32u + g * 8u;
      u32x4v x = {0u, 0u, 0u, 0u};
      if (live) x = *reinterpret_cast<const u32x4v*>(a.q + row * a.ld_q + (uint64_t)head * DH + d);
      q[s] = __builtin_bit_cast(bf16x8, x);
    }
    const float ks = (E4M3 && a.k_scale ? a.k_scale[kh] : 1.0f) * a.scale * 1.44269504088896f;

    f32x4 acc[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;

    // ---- where the keys are: 64 entries of the table in a register
    const int32_t* const table = a.tables + (uint64_t)seq * a.max_blocks;
    const uint32_t in_block = (1u << a.block_shift) - 1u;
    uint32_t held = 0xffffffffu;      // first entry of the 64
    int32_t entries = -1;
    auto block_of = [&](uint32_t pos) -> uint32_t {
      const uint32_t b = pos >> a.block_shift;
      if ((b & ~63u) != held) {
        held = b & ~63u;
        entries = held + lane < a.max_blocks ? table[held + lane] : -1;
      }
      return (uint32_t)__builtin_amdgcn_readlane(entries, (int)(b & 63u));
    };
    const int32_t last_tile = (k_end - 1) & ~15;
    // Loads a step's keys and values; returns a bit per tile, whether its block is in the pool.
    auto load = [&](Step& st, int32_t kb) -> uint32_t {
      uint32_t there = 0;
#pragma unroll
      for (int p = 0; p < KP; ++p) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t pos = (uint32_t)min(kb + p * 32 + t * 16, last_tile);
          uint32_t id = block_of(pos);
          const bool in = id < a.n_blocks;
          there |= (in ? 1u : 0u) << (2 * p + t);
          id = in ? id : 0u;
          const uint64_t at = ((((uint64_t)id * a.kv_heads + kh) << a.block_shift) + (pos & in_block)) * (uint64_t)(DH * ES);
          const unsigned char* kp = (const unsigned char*)a.k + at;
          const unsigned char* vp = (const unsigned char*)a.v + at;
          const uint32_t ko = col * (DH * ES) + g * 16u;
#pragma unroll
          for (int s = 0; s < Step::KL; ++s) st.k[p][t][s] = *reinterpret_cast<const u32x4v*>(kp + (ko + (uint32_t)s * 64u));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t vo = (4u * g + (uint32_t)j) * (DH * ES) + col * (VW * ES);
            if constexpr (Step::VD == 4) {
              const uint4 x = *reinterpret_cast<const uint4*>(vp + vo);
              uint32_t* o = st.v[p][4 * t + j];
              o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w;
            } else if constexpr (Step::VD == 2) {
              const uint2 x = *reinterpret_cast<const uint2*>(vp + vo);
              st.v[p][4 * t + j][0] = x.x; st.v[p][4 * t + j][1] = x.y;
            } else {
              st.v[p][4 * t + j][0] = *reinterpret_cast<const uint32_t*>(vp + vo);
            }
          }
        }
      }
      return there;
    };

    auto key_of = [&](int32_t kb, int p, int j) { return kb + p * 32 + (j >> 2) * 16 + (int32_t)(4u * g) + (j & 3); };
    auto work = [&](Step& st, int32_t kb, uint32_t there) {
      const bool whole = kb + (int32_t)STEP <= least && there == (1u << (2 * KP)) - 1u;
      f32x4 s[KP][2];
#pragma unroll
      for (int p = 0; p < KP; ++p)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            u32x4v x;
            if constexpr (E4M3) {
              const u32x4v raw = st.k[p][t][i / 2];
              const uint32_t r0 = raw[2 * (i & 1)], r1 = raw[2 * (i & 1) + 1];
              x = u32x4v{two_bf16(r0, false), two_bf16(r0, true), two_bf16(r1, false), two_bf16(r1, true)};
            } else {
              x = st.k[p][t][i];
            }
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), q[i], c, 0, 0, 0);
          }
          s[p][t] = c * ks;
        }
      if (!whole) {
#pragma unroll
        for (int p = 0; p < KP; ++p)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key_of(kb, p, 4 * t + j) >= sees || !(there >> (2 * p + t) & 1u)) s[p][t][j] = -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int p = 0; p < KP; ++p)
#pragma unroll
        for (int t = 0; t < 2; ++t) top = fmaxf(fmaxf(fmaxf(s[p][t][0], s[p][t][1]), fmaxf(s[p][t][2], s[p][t][3])), top);
      if (__any(top > m + 8.0f)) {           // m = -infinity: any key at all
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m2 = fmaxf(m, top), f = m2 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m2);
        l *= f;
#pragma unroll
        for (int i = 0; i < VW; ++i) acc[i] *= f;
        m = m2;
      }
      const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = __builtin_amdgcn_exp2f(s[p][j >> 2][j & 3] - base);
          l += e[j];
        }
        // p as bf16: 2^-8 of each term at most, in a sum of many; v has no more bits either
        const bf16x8 pk = __builtin_bit_cast(bf16x8, u32x4v{pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])});
        bool apart = false;
        if (!whole) {
          // 0 times what an unseen value holds is no 0 where that is NaN or infinite: nobody's positions become 0, and where
          // one that only some of the columns see is not finite, every column has its own product
          uint32_t odd = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int32_t key = key_of(kb, p, j);
            const bool seen = key < most && (there >> (2 * p + (j >> 2)) & 1u);
#pragma unroll
            for (int u = 0; u < Step::VD; ++u) {
              const uint32_t y = seen ? st.v[p][j][u] : 0u;
              st.v[p][j][u] = y;
              if (key >= least) odd |= not_finite<E4M3>(y);
            }
          }
          apart = least < most && __any(odd != 0);
        }
        // features 2 u and 2 u + 1 of a lane's VW: eight keys of two columns, two operands
        auto products = [&](int u, const uint32_t (&y)[8], f32x4& even, f32x4& uneven) {
          u32x4v lo, hi;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            lo[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], 0x05040100u);
            hi[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], 0x07060302u);
          }
          even = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pk, acc[2 * u], 0, 0, 0);
          uneven = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pk, acc[2 * u + 1], 0, 0, 0);
        };
        auto value = [&](int j, int u) { return E4M3 ? two_bf16(st.v[p][j][u / 2], u & 1) : st.v[p][j][u % Step::VD]; };
        if (!apart) {
#pragma unroll
          for (int u = 0; u < VW / 2; ++u) {
            uint32_t y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = value(j, u);
            products(u, y, acc[2 * u], acc[2 * u + 1]);
          }
        } else {
#pragma unroll 1
          for (uint32_t c = 0; c < n_cols; ++c) {
            const int32_t its = __builtin_amdgcn_readlane(sees, (int)c);
#pragma unroll
            for (int u = 0; u < VW / 2; ++u) {
              uint32_t y[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = key_of(kb, p, j) < its ? value(j, u) : 0u;
              f32x4 even, uneven;
              products(u, y, even, uneven);
              if (col == c) { acc[2 * u] = even; acc[2 * u + 1] = uneven; }
            }
          }
        }
      }
    };

    // ---- the keys, a step at a time, the next one's on their way meanwhile
    int32_t kb = k_first + (int32_t)(wave * STEP);
    if (kb < k_end) {
      Step one, two;
      uint32_t in_one = load(one, kb), in_two = 0;
      while (true) {
        if (kb + (int32_t)ROUND < k_end) in_two = load(two, kb + (int32_t)ROUND);
        work(one, kb, in_one);
        kb += (int32_t)ROUND;
        if (kb >= k_end) break;
        if (kb + (int32_t)ROUND < k_end) in_one = load(one, kb + (int32_t)ROUND);
        work(two, kb, in_two);
        kb += (int32_t)ROUND;
        if (kb >= k_end) break;
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // ---- the four wavefronts' sums together
    __syncthreads();                          // the last group's have been read
    if (g == 0) { sum_m[wave * COLS + col] = m; sum_l[wave * COLS + col] = l; }
    if (live) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < VW; i += 4)
          *reinterpret_cast<f32x4*>(sum_acc + (wave * COLS + col) * (DH + 4) + (4u * g + (uint32_t)j) * VW + (uint32_t)i) =
              f32x4{acc[i][j], acc[i + 1][j], acc[i + 2][j], acc[i + 3][j]};
    }
    __syncthreads();
    const float vs = E4M3 && a.v_scale ? a.v_scale[kh] : 1.0f;
    auto put = [&](uint32_t c, uint32_t d, const f32x4& o, float ls) {       // a column that saw nothing: zero
      const float inv = ls == 0.0f ? 0.0f : vs / ls;
      const uint32_t f = tile * COLS + c;
      bf16_t* to = a.out + (uint64_t)(w.row0 + f / a.group) * a.ld_out + (uint64_t)(kh * a.group + f % a.group) * DH + d;
      *reinterpret_cast<uint2*>(to) = ls == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    };
    constexpr uint32_t DV = DH / 4, STRIDE = DH + 4;
    auto part_of = [&](uint32_t place) { return parts + (uint64_t)place * part_cols * STRIDE; };
    for (uint32_t u = tid; u < n_cols * DV; u += 256) {
      const uint32_t c = u / DV, d = u % DV * 4u;
      Joined j;
#pragma unroll
      for (uint32_t x = 0; x < WAVES; ++x)
        j.add(sum_m[x * COLS + c], sum_l[x * COLS + c], *reinterpret_cast<const f32x4*>(sum_acc + (x * COLS + c) * STRIDE + d));
      if (pieces == 1) { put(c, d, j.o, j.l); continue; }
      float* to = part_of(2u * wg + (at_begin ? 0u : 1u)) + c * STRIDE;
      share_out(to + 4 + d, j.o[0], j.o[1]);
      share_out(to + 6 + d, j.o[2], j.o[3]);
      if (d == 0) share_out(to, j.m, j.l);
    }
    if (pieces == 1) continue;

    // ---- the last piece of a group to be done adds them up
    shared_out();
    __syncthreads();
    uint32_t* const arrived = (uint32_t*)red;
    if (tid == 0) {
      const uint32_t n = atomicAdd(counters + wg_first, 1u);
      if (n + 1u == pieces) __hip_atomic_store(counters + wg_first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      *arrived = n + 1u;
    }
    __syncthreads();
    if (*arrived != pieces) continue;
    const uint32_t first_place = 2u * wg_first + (group_first - SETUP <= share * wg_first ? 0u : 1u);
    const uint32_t lanes = n_cols * DV, teams = max(1u, 256u / lanes), team = tid / lanes;      // of threads, each with its pieces
    for (uint32_t u = tid % lanes; u < lanes && team < teams; u += 256) {
      const uint32_t c = u / DV, d = u % DV * 4u;
      Joined j;
#pragma unroll 4
      for (uint32_t x = team; x < pieces; x += teams) {
        const float* from = part_of(x ? 2u * (wg_first + x) : first_place) + c * STRIDE;
        const float2 ml = shared_in(from), lo = shared_in(from + 4 + d), hi = shared_in(from + 6 + d);
        j.add(ml.x, ml.y, f32x4{lo.x, lo.y, hi.x, hi.y});
      }
      if (teams == 1) { put(c, d, j.o, j.l); continue; }
      float* to = sum_acc + tid * 8u;
      *reinterpret_cast<f32x4*>(to) = j.o;
      to[4] = j.m; to[5] = j.l;
    }
    if (teams > 1) {
      __syncthreads();
      if (tid < lanes) {
        Joined j;
        for (uint32_t x = 0; x < teams; ++x) {
          const float* from = sum_acc + (x * lanes + tid) * 8u;
          j.add(from[4], from[5], *reinterpret_cast<const f32x4*>(from));
        }
        put(tid / DV, tid % DV * 4u, j.o, j.l);
      }
    }
  }
}

uint32_t part_columns(uint32_t n_rows, uint32_t group) { return (uint32_t)std::min<uint64_t>(COLS, (uint64_t)n_rows * group); }

template <int DH, bool E4M3>
hipError_t launch_paged(const PagedArgs& a, void* scratch, hipStream_t st) {
  constexpr int KP = E4M3 ? 2 : 1;
  const uint32_t rows = a.starts ? a.n_rows : std::min(a.n_rows, a.n_seq);
  if (rows == 0) return hipSuccess;
  uint32_t* counters = (uint32_t*)scratch;
  float* parts = (float*)scratch + MAX_WGS;
  const uint32_t lds = WAVES * COLS * (DH + 4) * 4 + WAVES * COLS * 8 + WAVES * 8 + (a.n_seq > 64 ? a.n_seq * 8 : 0);
  if (lds > 60u * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)paged_attention_kernel<DH, E4M3, KP>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  // units that there can be: column tiles, key heads, the longest sequence that the tables have room for
  const uint64_t tiles = ((uint64_t)rows * a.group + COLS - 1) / COLS + a.n_seq, units = (((uint64_t)a.max_blocks << a.block_shift) + UNIT - 1) / UNIT;
  const uint32_t wgs = (uint32_t)std::min<uint64_t>(MAX_WGS, (tiles * a.kv_heads * (units + SETUP) / MIN_SHARE + 8) / 8 * 8);
  paged_attention_kernel<DH, E4M3, KP><<<wgs, 256, lds, st>>>(a, counters, parts, part_columns(rows, a.group));
  return hipGetLastError();
}

}  // namespace

uint64_t paged_attention_scratch(uint32_t n_rows, uint32_t n_seq, uint32_t q_heads, uint32_t head_dim) {
  (void)n_seq;
  return MAX_WGS * 4 + 2ull * MAX_WGS * part_columns(n_rows, q_heads) * (head_dim + 4) * 4;
}

hipError_t launch_paged_attention(const PagedArgs& a, uint32_t head_dim, bool e4m3, void* scratch, hipStream_t st) {
  if (head_dim == 128) return e4m3 ? launch_paged<128, true>(a, scratch, st) : launch_paged<128, false>(a, scratch, st);
  return e4m3 ? launch_paged<64, true>(a, scratch, st) : launch_paged<64, false>(a, scratch, st);
}

}  // namespace qzo
