// Attention of the newest tokens of sequences over a paged cache where groups of them begin alike: the beams of a prompt, candidates behind
// one, a batch behind one long text.
//
// The keys that a group has in common are one item of work, with all the group's rows as its columns: they are read once, not once
// a sequence, and fill the matrix tiles that a single sequence leaves empty.  Every sequence's own keys are another item.  Both are
// the work of paged_attention_kernel (qzo_paged_kernel.hpp), which leaves (maximum m, sum l, accumulators o) of either; then
//   out = (o_c 2^(m_c - m) + o_s 2^(m_s - m)) / (l_c 2^(m_c - m) + l_s 2^(m_s - m)), m = max(m_c, m_s).
// A sequence that has nothing in common with its group writes its output itself.
#include "qzo_paged_kernel.hpp"

namespace qzo {
namespace {

// ---- common keys of many columns
// Nothing is masked here but what lies behind the last key, so a workgroup's eight wavefronts simply go through 64 keys at a time for 32
// columns each (256 in all; where a group's tile has at most 128, each column is two wavefronts', which take the keys in turns):
//   S[key][col]  = K Q^T      v_mfma_f32_32x32x16_bf16, K from the LDS
//   O[dim][col] += V^T P^T    P out of S's own registers: a lane holds column lane % 32 and keys 8 b + 4 (lane / 32) + 0..3, b = 0..3; two b's are the
//                             eight values of k that its place of the operand is to hold, if V's keys are dealt out the same way.
// Keys and values come through registers a step ahead; there an e4m3 one becomes bf16 and V is transposed (a thread four features of eight keys),
// once for all eight wavefronts.  16-byte pieces of a row change places in the LDS by the row's number, so that neighbouring rows are in
// different banks.
// The units of 64 keys of all groups, heads and tiles are dealt out in even shares; a tile's first piece leaves its share in place of its
// columns, a later one, with which its workgroup begins, in that workgroup's place; join_shares_kernel adds them up.
// An accumulator that is NaN, by a value whose weight is 0, say: the column is gone through again, one key a thread, without those.
// 64 sequences behind 32768 tokens, 64 heads on 8 of 128 (512 columns a key head, 69 GFLOP): 90 to 107 us, 650 to 770 TFLOP/s; matrix pipe busy 29 %
// of the SIMDs' time, vector pipe 37 %, no bank conflicts: two wavefronts a SIMD (64 accumulators, queries, scores, the values of a step and what is on
// its way: up to 255 registers with heads of 128), whose steps of loads from the LDS, products and weights overlap little.  The call 121 us, with paged_attention_kernel for this 217.
// 64 columns a wavefront would halve the LDS reads and do not fit (spills, 278 us for the call); priorities, four wavefronts a workgroup and a second
// step in registers gave nothing.  6 x 12 candidates of 9 tokens in e4m3, 40 heads on 8 of 64: 49 us (the call 82, otherwise 103), 1.2 to 2 us a step of 64 keys, most of them pieces' beginnings and ends.
// Weights meet the values rounded once to bf16: error against 64 bits as that of prompts, 2.0e-3 in the 2-norm, of which the output's rounding alone is
// 1.7e-3.  In two halves it is 1.7e-3, and the calls take 145 us in place of 122 and 86 in place of 83: not worth it.
constexpr uint32_t CK_THREADS = 512, CK_WAVES = 8, CK_KEYS = 64, CK_COLS = 32, CK_TILE = CK_COLS * CK_WAVES, CK_WGS = 256, CK_LEAST = 4;
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DH>
constexpr uint32_t ck_lds() { return std::max<uint32_t>(2 * 2 * CK_KEYS * DH * 2, CK_TILE / 2 * (DH + 4) * 4); }

template <int DH, bool E4M3>
__global__ __launch_bounds__(CK_THREADS, 2) void common_keys_kernel(SharedArgs a, float* parts) {
  constexpr uint32_t KS = DH / 16, MT = DH / 32, ROW = DH * 2, PIECES = ROW / 16, ES = E4M3 ? 1 : 2, STRIDE = DH + 4;
  constexpr uint32_t K_BYTES = CK_KEYS * ROW, BUFFER = 2 * K_BYTES;
  constexpr uint32_t K_LOADS = CK_KEYS * DH * ES / 16 / 256;            // 16-byte loads of a thread that sees to keys (the first 256 do)
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];   // two buffers of K and V^T, then what the groups are
  uint64_t* const first_unit = (uint64_t*)(lds + ck_lds<DH>());         // [n_groups + 1]
  int32_t* const group_starts = (int32_t*)(first_unit + a.n_groups + 1);  // [n_groups + 1]
  int32_t* const common = group_starts + a.n_groups + 1;                // [n_groups]
  int32_t* const leader = common + a.n_groups;                          // [n_groups]
  __shared__ uint64_t red[CK_WAVES];
  __shared__ uint32_t bad[CK_TILE];
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = scalar(tid >> 6), n = lane & 31u, hi = lane >> 5;

  // ---- the groups' units
  find_groups<CK_THREADS>(a, group_starts, common, leader);
  struct Group { uint32_t row0, cols, tiles, units; };
  auto group_of = [&](uint32_t g) {
    Group w;
    const uint32_t s0 = (uint32_t)group_starts[g], s1 = max(s0, (uint32_t)group_starts[g + 1]), end = row_of(a, s1);
    w.row0 = row_of(a, s0);
    w.cols = end > w.row0 ? (end - w.row0) * a.group : 0u;
    w.tiles = (w.cols + CK_TILE - 1) / CK_TILE;
    w.units = w.cols ? ((uint32_t)common[g] + CK_KEYS - 1) / CK_KEYS : 0u;
    return w;
  };
  const uint32_t per = (a.n_groups + CK_THREADS - 1) / CK_THREADS, g_first = min(tid * per, a.n_groups), g_end = min(g_first + per, a.n_groups);
  uint64_t mine = 0;
  for (uint32_t g = g_first; g < g_end; ++g) { const Group w = group_of(g); mine += (uint64_t)w.tiles * w.units * a.kv_heads; }
  uint64_t total = 0, before = 0;
  {
    uint64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t u = __shfl_up(upto, o, 64);
      if (lane >= (uint32_t)o) upto += u;
    }
    if (lane == 63u) red[wave] = upto;
    __syncthreads();
#pragma unroll
    for (uint32_t x = 0; x < CK_WAVES; ++x) { if (x < wave) before += red[x]; total += red[x]; }
    before += upto - mine;
  }
  for (uint32_t g = g_first; g < g_end; ++g) { const Group w = group_of(g); first_unit[g] = before; before += (uint64_t)w.tiles * w.units * a.kv_heads; }
  __syncthreads();
  total = scalar64(total);
  const uint64_t share = std::max<uint64_t>(CK_LEAST, (total + CK_WGS - 1) / CK_WGS);
  const uint32_t busy = (scalar((uint32_t)((total + share - 1) / share)) + 7u) / 8u * 8u;
  if (blockIdx.x >= busy) return;
  const uint32_t wg = (blockIdx.x & 7u) * (busy >> 3) + (blockIdx.x >> 3);           // neighbours on one XCD
  const uint64_t begin = share * wg, end = min(begin + share, total);

  for (uint64_t unit = begin; unit < end;) {
    uint32_t lo = 0, up = a.n_groups;
    while (up - lo > 1) {
      const uint32_t mid = (lo + up) >> 1;
      if (first_unit[mid] <= unit) lo = mid; else up = mid;
    }
    const uint32_t g = scalar(lo);
    Group w = group_of(g);
    w = {scalar(w.row0), scalar(w.cols), scalar(w.tiles), scalar(w.units)};
    const uint64_t r = scalar64(unit - first_unit[g]);
    const uint32_t which = scalar((uint32_t)(r / w.units)), at = scalar((uint32_t)(r - (uint64_t)which * w.units)), kh = scalar(which / w.tiles), tile = scalar(which % w.tiles);
    const uint32_t u_end = scalar((uint32_t)min((uint64_t)w.units, at + (end - unit)));
    const uint64_t group_end = unit - at + w.units;
    const uint32_t pieces = scalar((uint32_t)((group_end - 1) / share)) + 1u - wg;     // of the first piece's, this workgroup included
    unit += u_end - at;
    const uint32_t n_keys = scalar((uint32_t)common[g]), seq = scalar((uint32_t)leader[g]);

    // ---- this wavefront's columns
    const uint32_t col0 = tile * CK_TILE, n_cols = min(CK_TILE, w.cols - col0), blocks = (n_cols + CK_COLS - 1) / CK_COLS;
    const bool twice = blocks <= CK_WAVES / 2;
    const uint32_t cb = twice ? wave % (CK_WAVES / 2) : wave, part = twice ? wave / (CK_WAVES / 2) : 0u;
    const bool active = cb < blocks, live = cb * CK_COLS + n < n_cols;
    const uint32_t f = live ? col0 + cb * CK_COLS + n : col0, row = w.row0 + f / a.group, head = kh * a.group + f % a.group;
    bf16x8 q[KS];
    {
      const bf16_t* const from = a.q + (uint64_t)row * a.ld_q + (uint64_t)head * DH + hi * 8u;
#pragma unroll
      for (uint32_t s = 0; s < KS; ++s) {
        u32x4v x = *reinterpret_cast<const u32x4v*>(from + s * 16u);
        if (!live) x = u32x4v{0u, 0u, 0u, 0u};
        if (a.scale < 0.0f) x ^= 0x80008000u;
        q[s] = __builtin_bit_cast(bf16x8, x);
      }
    }
    const float ks = (E4M3 && a.k_scale ? a.k_scale[kh] : 1.0f) * fabsf(a.scale) * 1.44269504088896f;
    f32x16 o[MT];
#pragma unroll
    for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = -INFINITY, l = 0.0f;

    // ---- keys and values on their way: ids of a step's four 16-key tiles in scalar registers a step ahead of the loads
    const table_t table = (table_t)(uintptr_t)(a.tables + (uint64_t)seq * a.max_blocks);
    const uint32_t in_block = (1u << a.block_shift) - 1u, last16 = (n_keys - 1u) & ~15u;
    struct Ids { uint32_t id[4]; };
    auto ids_of = [&](uint32_t u) {
      Ids x;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) x.id[j] = (uint32_t)table[min(u * CK_KEYS + j * 16u, last16) >> a.block_shift];
      return x;
    };
    auto there_of = [&](uint32_t u, const Ids& x) {
      uint32_t there = 0;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) there |= u * CK_KEYS + j * 16u < n_keys && x.id[j] < a.n_blocks ? 1u << j : 0u;
      return there;
    };
    struct Staged { u32x4v k[4]; };
    auto load = [&](uint32_t u, const Ids& x) {
      Staged st;
      auto at_key = [&](uint32_t key, uint32_t id) {           // bytes from a pool's begin to the row of a key of the step
        const uint32_t pos = min(u * CK_KEYS + key, last16 + (key & 15u));
        return ((((uint64_t)(id < a.n_blocks ? id : 0u) * a.kv_heads + kh) << a.block_shift) + (pos & in_block)) * (uint64_t)(DH * ES);
      };
      if (wave < 4u) {
        constexpr uint32_t IN_ROW = DH * ES / 16;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          if (j >= K_LOADS) { st.k[j] = u32x4v{}; continue; }
          const uint32_t i = tid + 256u * j, key = i / IN_ROW;
          const uint32_t t = K_LOADS == 4 ? j : key >> 4, id = K_LOADS == 4 ? x.id[j] : t == 0 ? x.id[0] : t == 1 ? x.id[1] : t == 2 ? x.id[2] : x.id[3];
          st.k[j] = *reinterpret_cast<const u32x4v*>((const unsigned char*)a.k + at_key(key, id) + i % IN_ROW * 16u);
        }
      } else {
        // four features of eight keys: of tile t those 4 h + 0..3 and 8 more
        const uint32_t v = tid - 256u, four = v % (DH / 4), set = v / (DH / 4) % 8u, t = set >> 1, h = set & 1u;
        const uint32_t id = t == 0 ? x.id[0] : t == 1 ? x.id[1] : t == 2 ? x.id[2] : x.id[3];
        const unsigned char* const from = (const unsigned char*)a.v + at_key(t * 16u + 4u * h, id) + four * (4 * ES);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          const unsigned char* const x8 = from + (j < 4 ? j : j + 4u) * (DH * ES);
          uint32_t d0, d1;
          if constexpr (E4M3) {
            d0 = *reinterpret_cast<const uint32_t*>(x8); d1 = 0;
          } else {
            const uint2 y = *reinterpret_cast<const uint2*>(x8);
            d0 = y.x; d1 = y.y;
          }
          st.k[j / 2][j % 2 * 2] = d0;
          st.k[j / 2][j % 2 * 2 + 1] = d1;
        }
      }
      return st;
    };
    auto k_place = [](uint32_t key, uint32_t piece) { return key * ROW + (piece ^ (key & (PIECES - 1u))) * 16u; };
    auto v_place = [](uint32_t dim, uint32_t set) { return dim * (CK_KEYS * 2u) + (set ^ ((dim >> 2 ^ dim) & 7u)) * 16u; };
    auto store = [&](unsigned char* buffer, const Staged& st, uint32_t there) {
      if (wave < 4u) {
        constexpr uint32_t IN_ROW = DH * ES / 16;
#pragma unroll
        for (uint32_t j = 0; j < K_LOADS; ++j) {
          const uint32_t i = tid + 256u * j, key = i / IN_ROW, piece = i % IN_ROW;
          if constexpr (E4M3) {
            const u32x4v& x = st.k[j];
            *reinterpret_cast<u32x4v*>(buffer + k_place(key, 2u * piece)) = u32x4v{two_bf16(x[0], false), two_bf16(x[0], true), two_bf16(x[1], false), two_bf16(x[1], true)};
            *reinterpret_cast<u32x4v*>(buffer + k_place(key, 2u * piece + 1u)) = u32x4v{two_bf16(x[2], false), two_bf16(x[2], true), two_bf16(x[3], false), two_bf16(x[3], true)};
          } else {
            *reinterpret_cast<u32x4v*>(buffer + k_place(key, piece)) = st.k[j];
          }
        }
      } else {
        const uint32_t v = tid - 256u, four = v % (DH / 4), set = v / (DH / 4);
        if (set < 8u) {
          const bool here = there >> (set >> 1) & 1u;          // nobody's keys may hold anything
          uint32_t d[8][2];
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j) {
            uint32_t x = st.k[j / 2][j % 2 * 2], y = st.k[j / 2][j % 2 * 2 + 1];
            if constexpr (E4M3) { y = two_bf16(x, true); x = two_bf16(x, false); }
            d[j][0] = here ? x : 0u;
            d[j][1] = here ? y : 0u;
          }
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i) {
            u32x4v x;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_perm(d[2 * j + 1][i / 2], d[2 * j][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
            *reinterpret_cast<u32x4v*>(buffer + K_BYTES + v_place(four * 4u + i, set)) = x;
          }
        }
      }
    };

    // ---- 32 keys; their values come out of the LDS while the weights are computed
    auto work = [&](const unsigned char* buffer, uint32_t sub, uint32_t there) {
      f32x16 s;
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < KS; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(buffer + k_place(sub * 32u + n, 2u * i + hi)), q[i], s, 0, 0, 0);
      bf16x8 v[2][MT];
#pragma unroll
      for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
        for (uint32_t i = 0; i < MT; ++i) v[t][i] = *reinterpret_cast<const bf16x8*>(buffer + K_BYTES + v_place(i * 32u + n, sub * 4u + 2u * t + hi));
      const bool first16 = there >> (2u * sub) & 1u, second16 = there >> (2u * sub + 1u) & 1u;
      if (!(first16 && second16)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = (j < 8 ? first16 : second16) ? s[j] : -INFINITY;
      }
      float top = s[0];
#pragma unroll
      for (int j = 1; j < 15; j += 2) top = fmaxf(fmaxf(top, s[j]), s[j + 1]);
      top = fmaxf(top, s[15]) * ks;
      if (__any(top > m + 8.0f)) {               // m = -infinity: any key at all
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m2 = fmaxf(m, top), less = m2 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m2);
        l *= less;
#pragma unroll
        for (uint32_t i = 0; i < MT; ++i) o[i] *= less;
        m = m2;
      }
      const float base = m == -INFINITY ? 0.0f : m;
      bf16x8 p[2];
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float e[8];
        const bool seen = t ? second16 : first16;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + j], ks, -base));
          if (!seen) e[j] = 0.0f;                // (a scale of 0 times -infinity)
        }
        u32x4v x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t two = pack_bf16x2(e[2 * j], e[2 * j + 1]);
          x[j] = two;
          l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, l, false);      // the sum is that of what meets v
        }
        p[t] = __builtin_bit_cast(bf16x8, x);
      }
#pragma unroll
      for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
        for (uint32_t i = 0; i < MT; ++i)
          o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[t][i], p[t], o[i], 0, 0, 0);
    };

    __syncthreads();                              // what the last piece left in the LDS has been read
    Ids ids = ids_of(at);
    uint32_t there = there_of(at, ids);
    Staged st = load(at, ids);
    ids = ids_of(min(at + 1u, u_end - 1u));
    store(lds, st, there);
    __syncthreads();
    uint32_t buffer = 0;
#pragma unroll 1
    for (uint32_t u = at; u < u_end; ++u) {
      const uint32_t next = min(u + 1u, u_end - 1u), there_next = there_of(next, ids);      // (the last step again: without a branch around the loads)
      st = load(next, ids);
      ids = ids_of(min(next + 1u, u_end - 1u));
      if (active) {
#pragma unroll 1
        for (uint32_t sub = twice ? part : 0u; sub < (twice ? part + 1u : 2u); ++sub) work(lds + buffer * BUFFER, sub, there);
      }
      buffer ^= 1u;
      store(lds + buffer * BUFFER, st, there_next);
      there = there_next;
      __syncthreads();
    }
    l += __shfl_xor(l, 32, 64);

    // ---- two wavefronts' sums together
    if (twice) {
      float* const other = (float*)lds + (cb * CK_COLS + n) * STRIDE;
      if (part && active) {
        if (hi == 0) *reinterpret_cast<float2*>(other) = make_float2(m, l);
#pragma unroll
        for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
          for (uint32_t b = 0; b < 4; ++b) *reinterpret_cast<f32x4*>(other + 4 + i * 32u + b * 8u + hi * 4u) = f32x4{o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]};
      }
      __syncthreads();
      if (!part && active) {
        const float2 ml = *reinterpret_cast<const float2*>(other);
        const float top = fmaxf(m, ml.x), f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top), f1 = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);
        m = top;
        l = l * f0 + ml.y * f1;
#pragma unroll
        for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
          for (uint32_t b = 0; b < 4; ++b) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(other + 4 + i * 32u + b * 8u + hi * 4u);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][4 * b + j] = o[i][4 * b + j] * f0 + x[j] * f1;
          }
      }
    }
    // ---- the share of the common keys, or of a piece of them
    const bool writes = active && !part;
    auto place_of = [&](uint32_t f, uint32_t c) {      // column f of the group, c of the tile
      return at ? parts + ((uint64_t)wg * CK_TILE + c) * STRIDE
                : a.shares + ((uint64_t)a.n_rows * a.q_heads + (uint64_t)(w.row0 + f / a.group) * a.q_heads + kh * a.group + f % a.group) * STRIDE;
    };
    float all = l;
    if (writes) {
#pragma unroll
      for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) all += o[i][j];
    }
    const bool has_nan = writes && live && all != all;
    __syncthreads();
    if (writes && live) {
      const uint32_t c = cb * CK_COLS + n;
      float* const to = place_of(f, c);
      if (hi == 0) *reinterpret_cast<f32x4*>(to) = f32x4{m, l, __uint_as_float(wg << 16 | pieces), __uint_as_float(c)};      // (a first piece's: where the others are)
#pragma unroll
      for (uint32_t i = 0; i < MT; ++i)
#pragma unroll
        for (uint32_t b = 0; b < 4; ++b) *reinterpret_cast<f32x4*>(to + 4 + i * 32u + b * 8u + hi * 4u) = f32x4{o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]};
    }
    if (tid < CK_TILE) bad[tid] = 0;
    if (!__syncthreads_or(has_nan)) continue;
    if (has_nan) bad[cb * CK_COLS + n] = 1;
    __syncthreads();
    // ---- such columns again: a key a thread, then a feature a thread
    float* const weights = (float*)lds;           // [CK_THREADS]
    float* const tops = weights + CK_THREADS;     // [CK_WAVES]
    for (uint32_t c = 0; c < n_cols; ++c) {
      if (!bad[c]) continue;
      const uint32_t fc = col0 + c;
      const bf16_t* const qc = a.q + (uint64_t)(w.row0 + fc / a.group) * a.ld_q + (uint64_t)(kh * a.group + fc % a.group) * DH;
      auto row_at = [&](const void* pool, uint32_t pos, uint32_t id) {
        return (const unsigned char*)pool + ((((uint64_t)id * a.kv_heads + kh) << a.block_shift) + (pos & in_block)) * (uint64_t)(DH * ES);
      };
      auto value = [&](const unsigned char* r, uint32_t d) {
        if constexpr (E4M3) { const uint32_t x = two_bf16(r[d], false); return __uint_as_float(x << 16); }
        else return bf16_to_f32(reinterpret_cast<const bf16_t*>(r)[d]);
      };
      auto score = [&](uint32_t pos) {            // -infinity: not seen
        if (pos >= min(u_end * CK_KEYS, n_keys)) return -INFINITY;
        const uint32_t id = (uint32_t)table[pos >> a.block_shift];
        if (id >= a.n_blocks) return -INFINITY;
        const unsigned char* const r = row_at(a.k, pos, id);
        float x = 0.0f;
        for (uint32_t d = 0; d < DH; ++d) x = __builtin_fmaf(value(r, d), bf16_to_f32(qc[d]), x);
        return x == -INFINITY && a.scale > 0.0f ? x : x == INFINITY && a.scale < 0.0f ? -x : x * (a.scale < 0.0f ? -ks : ks);
      };
      float top = -INFINITY;
      for (uint32_t pos = at * CK_KEYS + tid; pos < u_end * CK_KEYS; pos += CK_THREADS) top = fmaxf(top, score(pos));
      top = wave_max(top);
      __syncthreads();
      if (lane == 0) tops[wave] = top;
      __syncthreads();
      for (uint32_t x = 0; x < CK_WAVES; ++x) top = fmaxf(top, tops[x]);
      const float base2 = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f, acc = 0.0f;
      for (uint32_t p0 = at * CK_KEYS; p0 < u_end * CK_KEYS; p0 += CK_THREADS) {
        const float x = score(p0 + tid);
        __syncthreads();
        weights[tid] = x == -INFINITY ? -1.0f : __uint_as_float(pack_bf16x2(__builtin_amdgcn_exp2f(x - base2), 0.0f) << 16);
        __syncthreads();
        for (uint32_t j = 0; j < CK_THREADS; ++j) {
          const float p = weights[j];
          if (p == -1.0f) continue;
          sum += p;
          if (tid < DH) acc = __builtin_fmaf(p, value(row_at(a.v, p0 + j, (uint32_t)table[(p0 + j) >> a.block_shift]), tid), acc);
        }
      }
      float* const to = place_of(fc, c);
      if (tid == 0) *reinterpret_cast<float2*>(to) = make_float2(top, sum);
      if (tid < DH) to[4 + tid] = acc;
    }
  }
}

// A row's head a team of DH / 4 lanes.
template <int DH>
__global__ __launch_bounds__(256) void join_shares_kernel(SharedArgs a, bool e4m3, const float* parts) {
  constexpr uint32_t LANES = DH / 4, STRIDE = DH + 4;
  const uint64_t pair = (uint64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const uint32_t row = (uint32_t)(pair / a.q_heads), head = (uint32_t)(pair % a.q_heads), d = threadIdx.x % LANES * 4u;
  uint32_t first = 0, end = min(a.n_seq, a.n_rows);
  if (a.starts) {
    first = (uint32_t)min(max(a.starts[0], 0), (int32_t)a.n_rows);
    end = (uint32_t)min(max(a.starts[a.n_seq], 0), (int32_t)a.n_rows);
  }
  if (row < first || row >= end) return;
  const float* const own = a.shares + pair * STRIDE;
  const float* const common = own + (uint64_t)a.n_rows * a.q_heads * STRIDE;
  const f32x4 head_own = *reinterpret_cast<const f32x4*>(own), head_common = *reinterpret_cast<const f32x4*>(common);
  const f32x4 o_own = *reinterpret_cast<const f32x4*>(own + 4 + d), o_common = *reinterpret_cast<const f32x4*>(common + 4 + d);
  if (head_own[2] == 0.0f) return;          // written already
  Joined j;
  j.add(head_common[0], head_common[1], o_common);
  if (parts) {                              // of common_keys_kernel: the pieces behind the first
    // (starts that do not ascend may leave a row without a common share: what is read then is at least a piece)
    const uint32_t where = __float_as_uint(head_common[2]), c = min(__float_as_uint(head_common[3]), CK_TILE - 1u);
    const uint32_t wg = min(where >> 16, CK_WGS - 1u), pieces = min(where & 0xffffu, CK_WGS - wg);
    for (uint32_t i = 1; i < pieces; i += 4) {
      float2 ml[4];
      f32x4 x[4];
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) {
        const float* const from = parts + ((uint64_t)(wg + min(i + k, pieces - 1u)) * CK_TILE + c) * STRIDE;
        ml[k] = *reinterpret_cast<const float2*>(from);
        x[k] = *reinterpret_cast<const f32x4*>(from + 4 + d);
      }
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k)
        if (i + k < pieces) j.add(ml[k].x, ml[k].y, x[k]);
    }
  }
  j.add(head_own[0], head_own[1], o_own);
  const float inv = (e4m3 && a.v_scale ? a.v_scale[head / a.group] : 1.0f) / j.l;
  bf16_t* const to = a.out + (uint64_t)row * a.ld_out + (uint64_t)head * DH + d;
  *reinterpret_cast<uint2*>(to) = j.l == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(j.o[0] * inv, j.o[1] * inv), pack_bf16x2(j.o[2] * inv, j.o[3] * inv));
}

// Columns that a group has on average from which on its common keys are common_keys_kernel's.  The call with paged_attention_kernel for them / with
// common_keys_kernel, us, 32 columns, 64, 96, 128; heads of 64: one group behind 1000 tokens 17 / 22, 17 / 23, 29 / 23, 32 / 24, one behind 32768 41 / 46, 41 / 47,
// 84 / 48, 154 / 49, 40 behind 1000 50 / 62, 82 / 74, 129 / 84, 165 / 96; heads of 128: 19 / 24, 19 / 25, 50 / 27, 56 / 28, then 66 / 51, 84 / 53, 153 / 56, 296 / 59,
// then 91 / 76, 152 / 96, 235 / 119, 242 / 141; in e4m3 much the same.  More than 64 columns always gain; fewer do where there are many keys, which the host does not know.
constexpr uint32_t CK_FROM = 65;
bool many_columns(uint32_t n_rows, uint32_t group, uint32_t n_groups) { return (uint64_t)n_rows * group >= (uint64_t)CK_FROM * n_groups; }
uint32_t shared_part_columns(uint32_t n_rows, uint32_t group) {
  return (uint32_t)std::min<uint64_t>(TILED_GROUP, (uint64_t)n_rows * group);
}
// Pieces of paged_attention_kernel, then those of common_keys_kernel.
uint64_t parts_bytes(uint32_t n_rows, uint32_t group, uint32_t head_dim) {
  const uint64_t own = 2ull * MAX_WGS * shared_part_columns(n_rows, group) * (head_dim + 4) * 4;
  return own + ((uint64_t)n_rows * group >= CK_FROM ? (uint64_t)CK_WGS * CK_TILE * (head_dim + 4) * 4 : 0);
}

// Items item_first .. item_first + n_items - 1.
template <int DH, bool E4M3, int CT, bool TILED>
hipError_t launch_items(SharedArgs a, uint32_t rows, uint32_t first, uint32_t n_items, void* scratch, hipStream_t st) {
  constexpr uint32_t TC = COLS * CT, GC = TILED ? TILED_GROUP : TC;
  a.item_first = first; a.n_items = n_items;
  uint32_t* counters = (uint32_t*)scratch;
  float* parts = (float*)scratch + MAX_WGS;
  const uint64_t groups = (2 * (((uint64_t)rows * a.group + GC - 1) / GC) + n_items) * a.kv_heads;
  const uint64_t units = (((uint64_t)a.max_blocks << a.block_shift) + 31) / 32;
  const bool few = n_items <= 64 && (double)groups * (double)(2 * units + 2) < 4e9;      // 32 bits hold the sums, padding included
  const uint32_t sums = WAVES * TC * (DH + 4) * 4 + WAVES * TC * 8, row = DH * (E4M3 ? 1u : 2u), tiles = TILED ? 8u * tile_step(row) * row : 0u;
  const uint32_t fixed = std::max(sums, tiles) + WAVES * 8, lds = fixed + (few ? 0 : n_items * 8) + (3 * a.n_groups + 1) * 4;
  if (lds > 60u * 1024) {                       // the limit that all calls have in common
    hipError_t e = hipFuncSetAttribute((const void*)paged_attention_kernel<DH, E4M3, CT, TILED, true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)(fixed + CACHE_MAX_SEQ * 8 + (3 * SHARED_MAX_GROUPS + 1) * 4));
    if (e != hipSuccess) return e;
  }
  const uint32_t wgs = (uint32_t)std::min<uint64_t>(MAX_WGS, (groups * ((units + MIN_PIECE - 1) / MIN_PIECE) + 7) / 8 * 8);
  const bool may_be_wide = !TILED && (uint64_t)rows * a.group > 2 * TC;
  paged_attention_kernel<DH, E4M3, CT, TILED, true><<<wgs, THREADS, lds, st>>>(a, counters, parts, shared_part_columns(a.n_rows, a.group), few, may_be_wide);
  return hipGetLastError();
}

// Items whose rows make `cols` columns a key head on average.
template <int DH, bool E4M3>
hipError_t launch_by_columns(const SharedArgs& a, uint32_t rows, double cols, uint32_t first, uint32_t n_items, void* scratch, hipStream_t st) {
  if (cols >= TILED_COLS) return launch_items<DH, E4M3, 2, true>(a, rows, first, n_items, scratch, st);
  if constexpr (many_tiles(DH) > 1)
    if (cols >= MANY_COLS) return launch_items<DH, E4M3, (int)many_tiles(DH), false>(a, rows, first, n_items, scratch, st);
  return launch_items<DH, E4M3, 1, false>(a, rows, first, n_items, scratch, st);
}

template <int DH, bool E4M3>
hipError_t launch_shared(SharedArgs a, void* scratch, hipStream_t st) {
  const uint32_t rows = a.starts ? a.n_rows : std::min(a.n_rows, a.n_seq);
  if (rows == 0) return hipSuccess;
  a.shares = (float*)((char*)scratch + MAX_WGS * 4 + parts_bytes(a.n_rows, a.group, DH));
  const double all = (double)rows * a.group, of_group = all / a.n_groups, of_seq = all / a.n_seq;
  float* pieces = nullptr;
  hipError_t e = hipSuccess;
  if (many_columns(rows, a.group, a.n_groups)) {
    pieces = (float*)((char*)scratch + MAX_WGS * 4) + 2ull * MAX_WGS * shared_part_columns(a.n_rows, a.group) * (DH + 4);
    const uint32_t lds = ck_lds<DH>() + (a.n_groups + 1) * 8 + (3 * a.n_groups + 1) * 4;
    e = hipFuncSetAttribute((const void*)common_keys_kernel<DH, E4M3>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(ck_lds<DH>() + (SHARED_MAX_GROUPS + 1) * 20));
    if (e != hipSuccess) return e;
    common_keys_kernel<DH, E4M3><<<CK_WGS, CK_THREADS, lds, st>>>(a, pieces);
    e = hipGetLastError();
    if (e == hipSuccess) e = launch_by_columns<DH, E4M3>(a, rows, of_seq, a.n_groups, a.n_seq, scratch, st);
  } else if (a.n_groups + a.n_seq > CACHE_MAX_SEQ) {
    e = launch_by_columns<DH, E4M3>(a, rows, of_group, 0, a.n_groups, scratch, st);
    if (e == hipSuccess) e = launch_by_columns<DH, E4M3>(a, rows, of_seq, a.n_groups, a.n_seq, scratch, st);
  } else {
    e = launch_by_columns<DH, E4M3>(a, rows, of_group, 0, a.n_groups + a.n_seq, scratch, st);
  }
  if (e != hipSuccess) return e;
  const uint64_t pairs = (uint64_t)a.n_rows * a.q_heads, per = 1024 / DH;
  join_shares_kernel<DH><<<(uint32_t)((pairs + per - 1) / per), 256, 0, st>>>(a, E4M3, pieces);
  return hipGetLastError();
}

}  // namespace

uint64_t paged_attention_shared_scratch(uint32_t n_rows, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim) {
  return MAX_WGS * 4 + parts_bytes(n_rows, q_heads / kv_heads, head_dim) + 2ull * n_rows * q_heads * (head_dim + 4) * 4;
}

hipError_t launch_paged_attention_shared(const SharedArgs& a, uint32_t head_dim, bool e4m3, void* scratch, hipStream_t st) {
  if (head_dim == 128) return e4m3 ? launch_shared<128, true>(a, scratch, st) : launch_shared<128, false>(a, scratch, st);
  return e4m3 ? launch_shared<64, true>(a, scratch, st) : launch_shared<64, false>(a, scratch, st);
}

}  // namespace qzo
