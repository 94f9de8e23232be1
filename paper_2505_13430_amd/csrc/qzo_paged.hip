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
// registers, eight 16-bit columns at a time, with one v_perm_b32 per pair of keys.  No LDS (but for prompts, below), no exchange between
// lanes but for the maximum, and that only when it has grown by a factor of 2^8: until then the sums carry the larger terms.
// All of a column's state (maximum, sum, its 4 VW accumulators) is in the lanes that hold the column.
//
// What bounds it: memory.  A step of a wavefront loads its next 32 keys (16 KB at heads of 128, bf16) before it works on the
// ones it has; eight wavefronts on a compute unit keep 128 to 256 KB on the way.  Loads and block ids are issued without a branch
// around them, or the compiler waits for all of them at every use.  8 sequences of 65536 tokens, 8 key heads of 128: 361 us,
// 5.9 TB/s (a kernel that only reads: 6.1 to 6.3); 64 ragged ones of up to 4001, 32 key heads, 150 to 156 us, 5.2 to 5.4 TB/s; 24 in
// e4m3 of up to 32001, 85 us, 4.9 TB/s (67 us at the reading kernel's rate).  Few keys: latency.  One token 7 us (launch, lengths,
// table, keys, one after the other); a compute unit alone takes 54 GB/s, 1.2 us a unit.
#include <algorithm>
#include <type_traits>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef const int32_t __attribute__((address_space(4)))* table_t;      // read by scalar loads: no vector load in between

// A wavefront has 16 columns; with heads of 64, for sequences of many columns (several new tokens; MANY_COLS on average), 32,
// two tiles that share the keys and the transposed values.  16 / 32 columns, us, 32 heads of 64: 16 prompts of 512 123 / 73, one
// 19 / 14, 6 x 100 tokens behind 1900 81 / 62, behind 900 44 / 38, 20 x 30 behind 970 63 / 50, 20 x 20 62 / 63.  (Heads of 128
// have no registers for it: with one step's keys and values in place of two, 277 us for the 144 of 6 x 100 tokens.)
//
// How the work is dealt out.  A group is a wavefront's columns of one sequence and key head; the four wavefronts of a workgroup
// take every fourth step (32 keys) of it, a unit is a step of each, 128 keys.  A wide group is four times those columns, a part
// for each wavefront, all with the same keys; a unit is then 32 keys.  It reads the keys once for the four and there are fewer
// groups, but it has a quarter of the loads on their way.  Narrow / wide, us, heads of 128: 16 prompts of 512 tokens (34816
// narrow units) 351 / 212, 6 x 100 tokens behind 1900 (21504) 194 / 144, 4 x 8 tokens, 64 heads on 8, behind 9000 (9088)
// 62 / 89, one prompt of 512 (4096) 32 / 43: wide from WIDE_UNITS on.  Heads of 64 with 32 columns, where there are few units
// a group: the prompts (4 of them) 130 / 73, but 6 x 100 tokens (16) 62 / 76, 4 x 200, 40 heads on 8 in e4m3 (32) 77 / 91.
//   Prompts (TILED): every group has 128 columns, 32 a wavefront, and the keys and values pass through the LDS, fetched once for the four
// and three steps ahead (32 keys a step where a row has 256 bytes, otherwise 64; rings of 64 KB, two workgroups a compute unit); a
// unit is 64 keys, a group ends with what its last column sees, and what is not cut goes to memory from the accumulators.  Without /
// so, us, heads of 128: 16 prompts of 512 tokens, 32 heads, 201 / 116, one of 2048 292 / 145, one of 4000 with 32 heads on 8 848 / 298 (440
// TFLOP/s), 4 x 200 tokens behind 3800, 40 heads on 8 in e4m3 181 / 145, 6 x 100 behind 1900 136 / 110, 4 of 130 (130 groups) 28 / 16,
// but one of 512 (128 groups) 31 / 32: from more groups than half the compute units on.  Heads of 64: one of 2048 (512 groups)
// 106 / 87, the prompts 76 / 61, but 4 x 200 in e4m3 (250) 89 / 96: from as many groups as workgroups on (6 x 100 behind 1900, 150 groups,
// 61 / 58, 9 x 100, 225, 65 / 63, 14 x 100, 350, 96 / 73: in bf16 from fewer on by now).  Fewer columns leave lanes idle: 4 x 8 tokens, 64
// heads on 8, behind 9000 (64 columns) 64 / 86, 20 x 40 behind 960 121 / 123: from TILED_COLS a sequence on.
// What bounds it: two wavefronts a SIMD, each a chain of LDS reads, products and exponentials (one of 4000: vector instructions 36 % of
// the time, matrix instructions 18 %; more steps ahead and LDS reads without conflicts did not make it faster, 16 % fewer vector
// instructions made it 6 % faster).  Heads of 128 have no registers left; what the compiler keeps in scratch memory is some
// 150 MB written in that call.
//   With more groups than workgroups, a sequence of up to QUAD_LEN positions and one wavefront's columns gives a workgroup four key heads at a time, one a
// wavefront (a unit is 32 keys of each): no other wavefront waits for a step that there is not, a workgroup starts a quarter
// as often, and nothing is added up in the end.  Such groups are not cut.  256 sequences, 32 heads of 128, of 1 / 20 / 64 /
// 128 / 300 / 500 positions: 76 / 83 / 91 / 129 / 236 / 380 us without, 35 / 45 / 61 / 107 / 229 / 375 so; 200 with 64 heads on
// 8 in e4m3: 24 / 24 / 25 / 29 / 46 / 60, so 13 / 14 / 16 / 20 / 37 / 53.  (64 ragged ones of up to 4001: 150, so 155; with
// QUAD_LEN 1024 169.)
//   Every group is given a span, its units behind some padding, all spans are counted through, and workgroup b takes those from
// share b to share (b + 1) - 1.
//   Few groups: the shortest piece that leaves no more pieces than workgroups is the share, and a span is a multiple of it, so
//     that every workgroup has one piece of one group, or nothing.
//   Otherwise: even shares whatever the lengths, a group's padding being SETUP, which stands for what a group costs apart from its
//     keys; a group no longer than an eighth of a share is not cut but belongs to whom its first unit falls to.
// A group that lies in one workgroup is written by it; otherwise each leaves (maximum, sum, accumulators) in the scratch, its
// first group's in place 2 b, a later one's (only the last can go on) in 2 b + 1, and who finds the group's counter at its last
// piece adds them up, in order.  The counter (that of the workgroup of the group's first piece) goes back to zero.
constexpr uint32_t COLS = 16, WAVES = 4, THREADS = 64 * WAVES, MAX_WGS = PAGED_COUNTERS;
constexpr uint32_t SETUP = 1, MIN_PIECE = 2, WIDE_UNITS = 12288, MANY_COLS = 24, QUAD_LEN = 512;
constexpr uint32_t TILE_KEYS = 64, TILED_GROUP = 2 * COLS * WAVES, TILED_PIECE = 8, TILED_COLS = 96;

// Keys that are waited for at a time where they go through the LDS: four times 16 KB, or 8 KB, are on their way or worked on.
constexpr uint32_t tile_step(uint32_t row) { return row == 256 ? 32u : 64u; }

struct SeqWork { uint32_t row0, rows, len, units, tiles, wide, quad; };

template <int CT, bool TILED>
struct Dealing {
  static constexpr uint32_t TC = COLS * CT;        // columns of a wavefront
  static __device__ __forceinline__ uint32_t unit(const SeqWork& w) { return TILED ? TILE_KEYS : w.wide || w.quad ? 32u : 32u * WAVES; }       // keys
  static __device__ __forceinline__ uint32_t heads(const SeqWork& w) { return w.quad ? WAVES : 1u; }      // key heads of a group
  static __device__ __forceinline__ uint32_t cols(const SeqWork& w) { return TILED || w.wide ? TC * WAVES : TC; }     // of a group
};

template <int CT, bool TILED>
__device__ __forceinline__ SeqWork seq_work(const PagedArgs& a, uint32_t i, bool wide, bool quads) {
  typedef Dealing<CT, TILED> D;
  SeqWork w;
  w.row0 = i; w.rows = i < a.n_rows ? 1u : 0u;
  if (a.starts) {
    const int32_t s0 = min(max(a.starts[i], 0), (int32_t)a.n_rows), s1 = min(max(a.starts[i + 1], s0), (int32_t)a.n_rows);
    w.row0 = (uint32_t)s0; w.rows = (uint32_t)(s1 - s0);
  }
  w.len = (uint32_t)min(max(a.lengths[i], 0), (int32_t)(a.max_blocks << a.block_shift));
  const uint64_t cols = (uint64_t)w.rows * a.group;
  w.wide = !TILED && wide && cols > 2 * D::TC;
  w.quad = !TILED && quads && cols <= D::TC && w.len <= QUAD_LEN;
  w.units = max(1u, (w.len + D::unit(w) - 1) / D::unit(w));
  w.tiles = (uint32_t)((cols + D::cols(w) - 1) / D::cols(w));
  return w;
}
// The column tiles of a key head, one after the other, and their units: TILED, those that the tile's last column sees, which in a
// prompt are fewer for the early ones.
template <bool TILED>
struct Tiles {
  const SeqWork& w;
  uint32_t group, step, rest, row = 0, part = 0, units;     // row, part: of the tile's first column, a token and a head of the group
  __device__ __forceinline__ Tiles(const PagedArgs& a, const SeqWork& w_) : w(w_), group(a.group), step(TILED_GROUP / a.group), rest(TILED_GROUP % a.group) { count(); }
  __device__ __forceinline__ void count() {
    if (!TILED) { units = w.units; return; }
    uint32_t last = row + step, beyond = part + rest;       // the next tile's first column; its token, or the one before, is the last
    if (beyond >= group) { beyond -= group; ++last; }
    if (beyond == 0) --last;
    const uint32_t after = w.rows - 1u - min(last, w.rows - 1u), sees = w.len > after ? w.len - after : 0u;
    units = max(1u, (sees + TILE_KEYS - 1) / TILE_KEYS);
  }
  __device__ __forceinline__ void next() {
    row += step; part += rest;
    if (part >= group) { part -= group; ++row; }
    count();
  }
};

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
__device__ __forceinline__ T block_scan(T v, T* total, T* red) {     // exclusive
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

// A step: 32 keys, two tiles.
template <int DH, bool E4M3>
struct PagedStep {
  static constexpr int KL = E4M3 ? DH / 64 : DH / 32;      // 16-byte loads a key tile takes
  static constexpr int VD = E4M3 ? DH / 64 : DH / 32;      // dwords of a row of V that a lane holds
  u32x4v k[2][KL];
  uint32_t v[8][VD];
};

template <int DH, bool E4M3, int CT, bool TILED>
__global__ __launch_bounds__(THREADS, 8 / WAVES) void paged_attention_kernel(PagedArgs a, uint32_t* counters, float* parts, uint32_t part_cols, uint32_t few, uint32_t may_be_wide) {
  constexpr int KS = DH / 32, VW = DH / 16, ES = E4M3 ? 1 : 2;
  typedef Dealing<CT, TILED> D;
  constexpr uint32_t TC = D::TC, STRIDE = DH + 4, ROW = DH * ES;
  typedef PagedStep<DH, E4M3> Step;
  constexpr int PARTS = DH == 64 && !E4M3 && !TILED ? 2 : 1;      // operands of bf16 that may hold a column's weights
  struct Weights { bf16x8 part[PARTS]; };
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  float* const sum_acc = (float*)lds;                                   // [WAVES][TC][STRIDE]; TILED: where the tiles were
  float* const sum_m = sum_acc + WAVES * TC * STRIDE;                   // [WAVES][TC]
  float* const sum_l = sum_m + WAVES * TC;
  constexpr uint32_t SUMS = WAVES * TC * (STRIDE + 2) * 4, TILES = TILED ? 8 * tile_step(ROW) * ROW : 0;
  uint64_t* const red = (uint64_t*)(lds + (SUMS > TILES ? SUMS : TILES));      // [WAVES]
  uint64_t* const first_unit = red + WAVES;                             // [n_seq], more than 64 sequences only
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = scalar(tid >> 6);
  const uint32_t col = lane & 15u, g = lane >> 4;

  // ---- the sequences' units: up to 64 sequences in the lanes of every wavefront, more in the LDS
  const uint32_t per = (a.n_seq + THREADS - 1) / THREADS, s_first = min(tid * per, a.n_seq), s_last = min(s_first + per, a.n_seq);
  SeqWork lane_work = {0, 0, 0, 1, 0, 0, 0};
  if (few && lane < a.n_seq) lane_work = seq_work<CT, TILED>(a, lane, false, false);
  bool wide = false, quads = false;
  auto sum = [&](auto&& f) -> uint64_t {            // of f over the sequences
    if (few) return (uint32_t)__builtin_amdgcn_readlane((int)lane_scan((uint32_t)f(lane_work)), 63);
    uint64_t n = 0, all;
    for (uint32_t i = s_first; i < s_last; ++i) n += f(seq_work<CT, TILED>(a, i, wide, quads));
    block_scan(n, &all, red);
    return scalar64(all);
  };
  auto head_groups = [&](const SeqWork& w) { return (a.kv_heads + D::heads(w) - 1) / D::heads(w); };
  auto groups_of = [&](const SeqWork& w) { return (uint64_t)w.tiles * head_groups(w); };
  // of a key head's tiles together: their units, or what f makes of them
  auto tiles_sum = [&](const SeqWork& w, auto&& f) -> uint64_t {
    if constexpr (!TILED) return (uint64_t)w.tiles * f(w.units);
    uint64_t n = 0;
    Tiles<TILED> its(a, w);
    for (uint32_t t = 0; t < w.tiles; ++t, its.next()) n += f(its.units);
    return n;
  };
  auto units_of = [&](const SeqWork& w) { return tiles_sum(w, [](uint32_t u) { return u; }) * head_groups(w); };
  uint64_t groups = sum(groups_of), units = sum(units_of);
  if (!TILED && may_be_wide && units >= WIDE_UNITS && (CT == 1 || units <= 8 * groups)) {
    wide = true;
    if (few && lane < a.n_seq) lane_work = seq_work<CT, TILED>(a, lane, true, false);
    groups = sum(groups_of); units = sum(units_of);
  }
  uint32_t piece = 0;                               // 0: even shares
  if (groups <= gridDim.x) {
    // Alone on its compute unit a workgroup takes 1.2 us a unit (heads of 128, bf16), the join of a cut group 3 to 4: pieces of
    // 2 units, but groups of up to 4 uncut.  One sequence, pieces of 1 / 2 / 3 / 4 units: 32 heads, 500 tokens 10.4 / 10.8 /
    // 11.8 / 10.5 us (heads of 64: 8.7 / 9.1 / 9.7 / 7.6), 1000 13.7 / 12.0 / 12.3 / 13.1, 4000 18.7 / 18.8 / 22.0 / 23.1; 8 key
    // heads, 4000 15.5 / 12.6 / 12.7 / 13.5, 16000 22.8 / 22.8 / 24.9 / 24.6.
    const uint32_t short_one = TILED ? TILED_PIECE : units <= 4 * groups ? 4u : MIN_PIECE;
    const uint32_t least = scalar(max(short_one, (uint32_t)((units + gridDim.x - 1) / gridDim.x))), more = max(1u, least / 16);
    for (uint32_t p = least; p < least + 3 * more && !piece; p += more)
      if (sum([&](const SeqWork& w) { return tiles_sum(w, [&](uint32_t u) { return (u + p - 1) / p; }) * head_groups(w); }) <= gridDim.x) piece = p;
  }
  if (!TILED && !piece) {
    quads = true;
    if (few && lane < a.n_seq) lane_work = seq_work<CT, TILED>(a, lane, wide, true);
  }
  auto span_of = [&](uint32_t u) { return piece ? (u + piece - 1) / piece * piece : u + SETUP; };
  auto head_span = [&](const SeqWork& w) { return tiles_sum(w, span_of); };
  uint64_t total;
  uint32_t mine = 0;
  if (few) {
    const uint32_t n = (uint32_t)(head_span(lane_work) * head_groups(lane_work)), upto = lane_scan(n);
    mine = upto - n;
    total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  } else {
    uint64_t n = 0;
    for (uint32_t i = s_first; i < s_last; ++i) {
      const SeqWork w = seq_work<CT, TILED>(a, i, wide, quads);
      first_unit[i] = n;
      n += head_span(w) * head_groups(w);
    }
    const uint64_t before = block_scan(n, &total, red);
    for (uint32_t i = s_first; i < s_last; ++i) first_unit[i] += before;
    __syncthreads();
    total = scalar64(total);
  }
  const uint64_t share = piece ? piece : (total + gridDim.x - 1) / gridDim.x;
  const uint32_t keep = piece ? 0u : (uint32_t)min(share / 8, (uint64_t)1 << 30);
  // those who have a share are spread over the XCDs, neighbours (the columns of the same keys) on one
  const uint32_t busy = scalar((uint32_t)((total + share - 1) / max(share, (uint64_t)1)) + 7u) / 8u * 8u;      // grid: a multiple of 8
  if (blockIdx.x >= busy) return;
  const uint32_t wg = (blockIdx.x & 7u) * (busy >> 3) + (blockIdx.x >> 3);
  const uint64_t begin = share * wg, end = min(begin + share, total);

  // the cut groups of this workgroup: the one that its share begins with, the one that it ends with
  struct Cut { uint32_t row0, group_col, kh, n_cols, wg_first, pieces, first_place; };
  Cut cut[2] = {};
  constexpr uint32_t DV = DH / 4;
  auto part_of = [&](uint32_t place) { return parts + (uint64_t)place * part_cols * STRIDE; };
  auto put = [&](uint32_t row0, uint32_t group_col, uint32_t kh, uint32_t c, uint32_t d, const Joined& j) {       // a column that saw nothing: zero
    const float inv = (E4M3 && a.v_scale ? a.v_scale[kh] : 1.0f) / j.l;
    const uint32_t f = group_col + c;
    bf16_t* to = a.out + (uint64_t)(row0 + f / a.group) * a.ld_out + (uint64_t)(kh * a.group + f % a.group) * DH + d;
    *reinterpret_cast<uint2*>(to) = j.l == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(j.o[0] * inv, j.o[1] * inv), pack_bf16x2(j.o[2] * inv, j.o[3] * inv));
  };

  // the last group's place: the next one's tile is looked for from there on
  uint32_t known_seq = ~0u, known_head = 0, known_tile = 0, known_row = 0, known_part = 0;
  uint64_t known_span = 0, known_before = 0;
  for (uint64_t unit = begin; unit < end;) {
    uint32_t seq;
    uint64_t seq_first;
    SeqWork w;
    if (few) {
      // prefixes ascend and begin at 0: the last one not above is the sequence that has the unit
      seq = scalar((uint32_t)__popcll(__ballot(lane < a.n_seq && mine <= (uint32_t)unit)) - 1u);
      auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)seq); };
      seq_first = of(mine);
      w = {of(lane_work.row0), of(lane_work.rows), of(lane_work.len), of(lane_work.units), of(lane_work.tiles), of(lane_work.wide), of(lane_work.quad)};
    } else {
      uint32_t lo = 0, hi = a.n_seq;
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first_unit[mid] <= unit) lo = mid; else hi = mid;
      }
      seq = scalar(lo);
      seq_first = scalar64(first_unit[seq]);
      w = seq_work<CT, TILED>(a, seq, wide, quads);
      w = {scalar(w.row0), scalar(w.rows), scalar(w.len), scalar(w.units), scalar(w.tiles), scalar(w.wide), scalar(w.quad)};
    }
    const uint64_t r = unit - seq_first;
    uint32_t tile, head, at;                                                  // at: within the group's span
    if constexpr (TILED) {
      if (seq != known_seq) { known_seq = seq; known_head = ~0u; known_span = scalar64(head_span(w)); }
      head = scalar((r >> 32) ? (uint32_t)(r / known_span) : (uint32_t)r / (uint32_t)known_span);
      const uint64_t rest = r - head * known_span;
      Tiles<TILED> its(a, w);
      if (head == known_head) {
        its.row = known_row; its.part = known_part; its.count();
      } else {
        known_head = head; known_tile = 0; known_before = 0;
      }
      while (rest >= known_before + span_of(its.units)) {
        known_before += span_of(its.units);
        ++known_tile;
        its.next();
      }
      known_row = scalar(its.row); known_part = scalar(its.part); known_tile = scalar(known_tile); known_before = scalar64(known_before);
      tile = known_tile; at = scalar((uint32_t)(rest - known_before));
      w.units = scalar(its.units);
    } else {
      const uint32_t s1 = scalar(span_of(w.units)), group = scalar((r >> 32) ? (uint32_t)(r / s1) : (uint32_t)r / s1);
      tile = scalar(group % w.tiles); head = scalar(group / w.tiles);
      at = scalar((uint32_t)(r - (uint64_t)group * s1));
    }
    const uint32_t span = scalar(span_of(w.units)), pad = span - w.units;
    const uint32_t kh0 = scalar(head * D::heads(w)), kh = kh0 + (w.quad ? wave : 0u);
    const bool uncut = span <= keep || w.quad;
    if (uncut && at) { unit += span - at; continue; }
    const uint32_t n_units = uncut ? span : scalar((uint32_t)min((uint64_t)(span - at), end - unit));
    const uint64_t group_first = unit - at + pad, group_last = unit - at + span - 1;
    const bool at_begin = unit == begin;
    unit += n_units;
    if (at + n_units <= pad) continue;
    const uint32_t u_first = max(at, pad) - pad, u_end = at + n_units - pad;
    uint32_t wg_first = wg, pieces = 1;
    if (!uncut) {
      if (group_first < begin) wg_first = wg - scalar((uint32_t)((begin - group_first + share - 1) / share));
      pieces = wg + 1u - wg_first;
      if (group_last >= end) pieces += scalar((uint32_t)((group_last - end) / share)) + 1u;
    }

    // ---- this wavefront's columns
    const uint32_t all_cols = w.rows * a.group, group_col = tile * D::cols(w), n_group = min(D::cols(w), all_cols - group_col);
    const uint32_t first_col = group_col + (TILED || w.wide ? wave * TC : 0u), n_cols = first_col < all_cols && kh < a.kv_heads ? min(TC, all_cols - first_col) : 0u;
    // Up to half the columns: lanes col and col + 8 have the same one, the first its weights in bf16, the second what their rounding left.
    const bool twice = CT == 1 && !TILED && n_group <= COLS / 2;
    const uint32_t own = twice ? col % (COLS / 2) : col;
    bool live[CT];
    // positions that a column sees, that the first (the fewest) and the last (the most) of them see
    int32_t sees[CT];
    const int32_t least = (int32_t)(w.len + first_col / a.group + 1u - w.rows);
    const int32_t most = n_cols ? (int32_t)(w.len + (first_col + n_cols - 1) / a.group + 1u - w.rows) : 0;
    const int32_t k_first = (int32_t)(u_first * D::unit(w)), k_end = (int32_t)min((int64_t)most, (int64_t)u_end * D::unit(w));
    // of all the group's columns
    const int32_t group_end = !TILED ? k_end : (int32_t)min((int64_t)w.len + (group_col + n_group - 1) / a.group + 1 - w.rows, (int64_t)u_end * TILE_KEYS);
    bf16x8 q[CT][KS];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      live[ct] = ct * COLS + own < n_cols;
      const uint32_t flat = live[ct] ? first_col + ct * COLS + own : group_col, token = flat / a.group, head = kh * a.group + flat % a.group;
      sees[ct] = live[ct] ? (int32_t)(w.len + token + 1u - w.rows) : 0;
      const bf16_t* from = a.q + (uint64_t)(w.row0 + token) * a.ld_q + (uint64_t)head * DH;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        // e4m3: a 16-byte load of K is two operands
        const uint32_t d = E4M3 ? (uint32_t)(s / 2) * 64u + g * 16u + (uint32_t)(s & 1) * 8u : (uint32_t)s * 32u + g * 8u;
        u32x4v x = {0u, 0u, 0u, 0u};
        if (live[ct]) x = *reinterpret_cast<const u32x4v*>(from + d);
        if (a.scale < 0.0f) x ^= 0x80008000u;
        q[ct][s] = __builtin_bit_cast(bf16x8, x);
      }
    }
    const float ks = (E4M3 && a.k_scale && n_cols ? a.k_scale[kh] : 1.0f) * fabsf(a.scale) * 1.44269504088896f;

    f32x4 acc[CT][VW];
    typedef std::conditional_t<TILED, f32x4, float> Sum;       // TILED: a matrix product's, four times the same
    float m[CT];
    Sum l[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int i = 0; i < VW; ++i) acc[ct][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      m[ct] = -INFINITY; l[ct] = Sum{};
    }

    // ---- where the keys are: a block id per tile, in scalar registers, a step ahead of the loads that need it
    const table_t table = (table_t)(uintptr_t)(a.tables + (uint64_t)seq * a.max_blocks);
    const uint32_t in_block = (1u << a.block_shift) - 1u;
    const int32_t last_tile = max(group_end - 1, 0) & ~15;       // steps beyond the end load it again (a branch around loads would have
                                                             // every wait count as if they had not been issued)
    struct Ids { uint32_t id[2]; };
    auto blocks = [&](int32_t kb) {
      return Ids{{(uint32_t)table[(uint32_t)min(kb, last_tile) >> a.block_shift], (uint32_t)table[(uint32_t)min(kb + 16, last_tile) >> a.block_shift]}};
    };
    auto present = [&](const Ids& ids) { return (ids.id[0] < a.n_blocks ? 1u : 0u) | (ids.id[1] < a.n_blocks ? 2u : 0u); };     // blocks of the pool
    auto load = [&](Step& st, int32_t kb, const Ids& ids) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t pos = (uint32_t)min(kb + t * 16, last_tile), id = ids.id[t] < a.n_blocks ? ids.id[t] : 0u;
        const uint64_t at = ((((uint64_t)id * a.kv_heads + kh) << a.block_shift) + (pos & in_block)) * (uint64_t)(DH * ES);
        const unsigned char* kp = (const unsigned char*)a.k + at;
        const unsigned char* vp = (const unsigned char*)a.v + at;
        const uint32_t ko = col * (DH * ES) + g * 16u;
#pragma unroll
        for (int s = 0; s < Step::KL; ++s) st.k[t][s] = *reinterpret_cast<const u32x4v*>(kp + (ko + (uint32_t)s * 64u));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t vo = (4u * g + (uint32_t)j) * (DH * ES) + col * (VW * ES);
          uint32_t* o = st.v[4 * t + j];
          if constexpr (Step::VD == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(vp + vo);
            o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w;
          } else if constexpr (Step::VD == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(vp + vo);
            o[0] = x.x; o[1] = x.y;
          } else {
            o[0] = *reinterpret_cast<const uint32_t*>(vp + vo);
          }
        }
      }
    };

    auto key_of = [&](int32_t kb, int j) { return kb + (j >> 2) * 16 + (int32_t)(4u * g) + (j & 3); };
    auto whole_step = [&](int32_t kb, uint32_t there) { return kb + 32 <= least && there == 3u; };       // every column sees all of it
    auto scores = [&](const Step& st, f32x4 (&s)[CT][2]) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) s[ct][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          u32x4v x;
          if constexpr (E4M3) {
            const uint32_t r0 = st.k[t][i / 2][2 * (i & 1)], r1 = st.k[t][i / 2][2 * (i & 1) + 1];
            x = u32x4v{two_bf16(r0, false), two_bf16(r0, true), two_bf16(r1, false), two_bf16(r1, true)};
          } else {
            x = st.k[t][i];
          }
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) s[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), q[ct][i], s[ct][t], 0, 0, 0);
        }
      }
    };
    // The weight 0 of a key that a column does not see, by its position or by a score of -infinity, does not keep out a value that is NaN
    // or infinite.  A step that has such a key is looked at (look); its scores tell, eight instructions.  TILED, where vector instructions
    // count, does not ask: with such a value a sum is NaN, and where one is at the end all keys are gone through once more, every step
    // looked at, with the same results everywhere else.  Asked / so, us: one prompt of 4000 325 / 298, 4 x 200 tokens in e4m3 184 / 144, 16
    // prompts of 512 with heads of 64 68 / 61.
    // s becomes p, as the second product's operand; the sums follow.  look: the weight of a key that its column does not see is -0
    // (UNSEEN), all others' have no sign.
    constexpr uint32_t UNSEEN = 0x8000u;
    auto softmax = [&](int ct, f32x4 (&s)[2], int32_t kb, uint32_t there, bool& look) {
      float f = ks;                             // TILED: the factor meets s in the exponential's own operand, but where a product with
      if (!TILED || !whole_step(kb, there)) {   // what stands for unseen might be none
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] *= ks;
        f = 1.0f;
        if (!whole_step(kb, there)) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (key_of(kb, j) >= sees[ct] || !(there >> (j >> 2) & 1u)) s[j >> 2][j & 3] = -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * f;
      if (__any(top > m[ct] + 8.0f)) {           // m = -infinity: any key at all
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m2 = fmaxf(m[ct], top), less = m2 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[ct] - m2);
        l[ct] *= less;
#pragma unroll
        for (int i = 0; i < VW; ++i) acc[ct][i] *= less;
        m[ct] = m2;
      }
      bool some_unseen = look;
      if constexpr (!TILED) {
        const float low = fminf(fminf(fminf(s[0][0], s[0][1]), fminf(s[0][2], s[0][3])), fminf(fminf(s[1][0], s[1][1]), fminf(s[1][2], s[1][3])));
        some_unseen = __any(low == -INFINITY);
        look |= some_unseen;
      }
      const float base = m[ct] == -INFINITY ? 0.0f : m[ct];
      float e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(s[j >> 2][j & 3], f, -base));
      // p as bf16, which the matrix instructions ask for: 2^-8 of each term at most; the sum is that of the rounded ones, so that what
      // rounds all weights alike, a key that takes all, cancels.  What is left of p goes into the idle half of the columns where there
      // is one (single tokens, up to eight heads a key head): 2^-16, at no cost (8 x 65536 tokens 362 us, 64 ragged 150, either way).
      // Otherwise it takes a second product for every value, which heads of 64 have the registers for (bf16: 6 x 100 tokens 49 / 51 us,
      // behind 1900 60 / 61, 20 x 30 behind 970 40.0 / 40.3; e4m3, whose values have been rounded by up to 2^-4, 4 x 200 behind 3800 79 /
      // 91: once).  Heads of 128 have not (4 x 8 tokens, 64 heads on 8, behind 9000 56 / 60, but single tokens, the same code, lose
      // their loads ahead: 64 ragged 152 / 181), and prompts are bound by such instructions (16 of 512 116 / 136, one of 4000 317 /
      // 379): those keep the one rounding, as the whole-sequence kernel does.
      u32x4v pk = {pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])};
      if (twice) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t rest = pack_bf16x2(e[2 * j] - __uint_as_float(pk[j] << 16), e[2 * j + 1] - __uint_as_float(pk[j] & 0xffff0000u));
          pk[j] = col < COLS / 2 ? pk[j] : rest;
        }
      }
      if (some_unseen) {
#pragma unroll
        for (int j = 0; j < 8; ++j) pk[j >> 1] |= s[j >> 2][j & 3] * f == -INFINITY ? UNSEEN << 16 * (j & 1) : 0u;
      }
      if constexpr (TILED) {                     // ones times p: every lane of the column has the sum of all
        const u32x4v ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, pk), l[ct], 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) l[ct] += PARTS > 1 && !twice ? e[2 * j] + e[2 * j + 1] : __uint_as_float(pk[j] << 16) + __uint_as_float(pk[j] & 0xffff0000u);
      }
      Weights p;
      p.part[0] = __builtin_bit_cast(bf16x8, pk);
      if constexpr (PARTS > 1) {
        u32x4v rest;
#pragma unroll
        for (int j = 0; j < 4; ++j) rest[j] = pack_bf16x2(e[2 * j] - __uint_as_float(pk[j] << 16), e[2 * j + 1] - __uint_as_float(pk[j] & 0xffff0000u));
        p.part[1] = __builtin_bit_cast(bf16x8, rest);
      }
      return p;
    };
    auto values = [&](Step& st, const Weights (&pk)[CT], int32_t kb, uint32_t there, bool look) {
      bool apart = false;
      if (look || !whole_step(kb, there)) {
        // nobody's positions, which may hold anything, become 0; where what is left is not finite, every column has its own product
        uint32_t odd = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool seen = key_of(kb, j) < most && (there >> (j >> 2) & 1u);
#pragma unroll
          for (int u = 0; u < Step::VD; ++u) {
            const uint32_t y = seen ? st.v[j][u] : 0u;
            st.v[j][u] = y;
            if (!TILED || look) odd |= not_finite<E4M3>(y);
          }
        }
        apart = __any(odd != 0);
      }
      // features 2 u and 2 u + 1 of a lane's VW: eight keys of two rows of V^T, two operands
      auto operand = [&](const uint32_t (&y)[8], uint32_t pick) {
        u32x4v o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], pick);
        return __builtin_bit_cast(bf16x8, o);
      };
      auto value = [&](int j, int u) { return E4M3 ? two_bf16(st.v[j][u / 2], u & 1) : st.v[j][u % Step::VD]; };
      if (!apart) {
#pragma unroll
        for (int u = 0; u < VW / 2; ++u) {
          uint32_t y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = value(j, u);
          const bf16x8 even = operand(y, 0x05040100u), uneven = operand(y, 0x07060302u);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int x = 0; x < PARTS; ++x) {
              if (x && twice) break;
              acc[ct][2 * u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pk[ct].part[x], acc[ct][2 * u], 0, 0, 0);
              acc[ct][2 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(uneven, pk[ct].part[x], acc[ct][2 * u + 1], 0, 0, 0);
            }
          }
        }
      } else {
        // (TILED: a pair of features at a time, so that few registers hold what is not in place)
        auto pair = [&](int ct, int u, uint32_t c) {
          uint32_t y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t p = (uint32_t)__shfl((int)__builtin_bit_cast(u32x4v, pk[ct].part[0])[j >> 1], (int)((lane & 48u) | c), 64);
            y[j] = (p >> 16 * (j & 1) & 0xffffu) == UNSEEN ? 0u : value(j, u);
          }
          f32x4 even = acc[ct][2 * u], uneven = acc[ct][2 * u + 1];
#pragma unroll
          for (int x = 0; x < PARTS; ++x) {
            if (x && twice) break;
            even = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(y, 0x05040100u), pk[ct].part[x], even, 0, 0, 0);
            uneven = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(y, 0x07060302u), pk[ct].part[x], uneven, 0, 0, 0);
          }
          if (col == c) { acc[ct][2 * u] = even; acc[ct][2 * u + 1] = uneven; }
        };
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if constexpr (TILED) {
#pragma unroll
            for (int u = 0; u < VW / 2; ++u)
#pragma unroll 1
              for (uint32_t c = 0; c < COLS; ++c) pair(ct, u, c);
          } else {
#pragma unroll 1
            for (uint32_t c = 0; c < COLS; ++c)
#pragma unroll
              for (int u = 0; u < VW / 2; ++u) pair(ct, u, c);
          }
        }
      }
    };

    auto work = [&](Step& st, int32_t kb, uint32_t there) {
      f32x4 s[CT][2];
      Weights pk[CT];
      bool look = false;
      scores(st, s);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) pk[ct] = softmax(ct, s[ct], kb, there, look);
      values(st, pk, kb, there, look);
    };
    if constexpr (TILED) {
      auto go_through = [&](auto careful) __attribute__((always_inline)) {       // careful: look at every step
        // ---- 32 or 64 keys at a time through the LDS, the next three such steps on their way.  A wavefront fetches a tile of 16 keys, lane by
        // lane 16 bytes to consecutive places; a row's 16-byte pieces change places there, so that lanes that read the same piece of 16
        // rows find it in different banks (256 bytes a row: K piece ^ row, V, whose rows are read as they lie, as they are; with
        // row & 7 for both half of all LDS cycles were conflicts).
        constexpr uint32_t KEYS = tile_step(ROW), TILE = 16 * ROW, HALF = KEYS * ROW, LOADS = TILE / 1024, BUFFERS = 4;
        constexpr bool BOTH = KEYS == 64;         // a wavefront fetches a tile of keys and one of values, not one of them
        auto turn = [](uint32_t row) { return ROW == 256 ? row : ROW == 128 ? row & 7u : row >> 1 & 3u; };
        uint32_t from[LOADS];
#pragma unroll
        for (uint32_t n = 0; n < LOADS; ++n) {
          const uint32_t byte = n * 1024u + lane * 16u, row = byte / ROW, piece16 = byte % ROW / 16u;
          from[n] = row * ROW + (BOTH || wave < 2u ? piece16 ^ turn(row) : piece16) * 16u;
        }
        const uint32_t own = BOTH ? wave : wave & 1u;            // its tile
        const uint32_t to = scalar((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + own * TILE + (BOTH ? 0u : (wave >> 1) * HALF));
        // block ids of 64 tiles in the lanes, those of the next 64 on their way; seen: which of them are in the pool
        const int32_t* const ids_at = a.tables + (uint64_t)seq * a.max_blocks;
        int32_t ids_from = k_first;
        auto ids_load = [&](int32_t kb) { return (uint32_t)ids_at[min((uint32_t)kb + 16u * lane, (uint32_t)last_tile) >> a.block_shift]; };
        uint32_t ids = ids_load(ids_from), ids_next = ids_load(ids_from + 1024);
        uint64_t seen = __ballot(ids < a.n_blocks);
        auto fetch = [&](uint32_t buffer, int32_t kb, uint32_t id) {
          const uint32_t pos = (uint32_t)min(kb + (int32_t)(own * 16u), last_tile);
          const uint64_t at16 = ((((uint64_t)(id < a.n_blocks ? id : 0u) * a.kv_heads + kh) << a.block_shift) + (pos & in_block)) * (uint64_t)ROW;
          typedef int i32x4 __attribute__((ext_vector_type(4)));
          auto tile_of = [&](const void* pool) {
            const uint64_t x = scalar64((uint64_t)(uintptr_t)pool + at16);
            return i32x4{(int)(uint32_t)x, (int)(uint32_t)(x >> 32), (int)TILE, 0x00020000};
          };
          const i32x4 first = tile_of(BOTH || wave < 2u ? a.k : a.v), second = tile_of(a.v);
#pragma unroll
          for (uint32_t n = 0; n < LOADS; ++n) {
            asm volatile(QZO_SET_M0 "buffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to + buffer * (2u * HALF) + n * 1024u), "v"(from[n]), "s"(first) : "memory", "m0");
            if constexpr (BOTH)
              asm volatile(QZO_SET_M0 "buffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to + buffer * (2u * HALF) + HALF + n * 1024u), "v"(from[n]), "s"(second) : "memory", "m0");
          }
        };
        const uint32_t k_at = col * ROW + (g ^ turn(col)) * 16u;
        uint32_t v_at[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) v_at[j] = (4u * g + j) * ROW + (col * (VW * ES) ^ (BOTH ? turn(4u * g + j) * 16u : 0u));
        __syncthreads();                          // what the last group left here has been read
        __builtin_amdgcn_s_waitcnt(0x0F70);       // vmcnt(0): the queries, or the compiler would wait for them, and for the next keys, below
        uint64_t there_of = 0;                    // of the steps on their way, 16 bits each, the newest lowest
        auto fetch_next = [&](uint32_t buffer, int32_t kb) {
          if (kb - ids_from >= 1024) {
            ids_from += 1024;
            ids = ids_next;
            seen = __ballot(ids < a.n_blocks);
            ids_next = ids_load(ids_from + 1024);
          }
          const uint32_t tile16 = (uint32_t)(kb - ids_from) >> 4;
          there_of = there_of << 16 | ((uint32_t)(seen >> tile16) & 15u);
          fetch(buffer, kb, (uint32_t)__builtin_amdgcn_readlane((int)ids, (int)(tile16 + own)));
        };
#pragma unroll
        for (uint32_t i = 0; i < BUFFERS - 1; ++i)
          if (k_first + (int32_t)(i * KEYS) < group_end) fetch_next(i, k_first + (int32_t)(i * KEYS)); else there_of <<= 16;
        uint32_t buffer = 0;
#pragma unroll 1
        for (int32_t kb = k_first; kb < group_end; kb += (int32_t)KEYS) {
          const uint32_t there = (uint32_t)(there_of >> 16 * (BUFFERS - 2)) & 15u;
          // this wavefront's part has come, the next two steps' may be on their way; behind the barrier all four parts have
          constexpr int STEP_LOADS = (int)(BOTH ? 2 * LOADS : LOADS);
          if (kb + 2 * (int32_t)KEYS < group_end) __builtin_amdgcn_s_waitcnt(0x0F70 | 2 * STEP_LOADS);
          else __builtin_amdgcn_s_waitcnt(0x0F70);
          __syncthreads();                        // and the step before has been read
          if (kb + (int32_t)((BUFFERS - 1) * KEYS) < group_end) fetch_next((buffer + BUFFERS - 1) % BUFFERS, kb + (int32_t)((BUFFERS - 1) * KEYS));
          else there_of <<= 16;
          const unsigned char* const tiles = lds + buffer * (2u * HALF);
          buffer = (buffer + 1) % BUFFERS;
#pragma unroll
          for (int part = 0; part < (int)KEYS / 32; ++part) {
            if (kb + 32 * part >= k_end) break;
            Step st;
            f32x4 s[CT][2];
            Weights pk[CT];
            bool look = careful;
            const int32_t k32 = kb + 32 * part;
            const uint32_t there32 = there >> (2 * part) & 3u;
            const unsigned char* const kt = tiles + 2 * part * TILE;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int i = 0; i < Step::KL; ++i) st.k[t][i] = *reinterpret_cast<const u32x4v*>(kt + t * TILE + (k_at ^ (uint32_t)i * 64u));
            scores(st, s);
            if (DH == 128) __builtin_amdgcn_sched_barrier(0);     // the values take the keys' registers
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t* o = st.v[j];
              const unsigned char* const vt = kt + HALF + (j >> 2) * TILE + v_at[j & 3];
              if constexpr (Step::VD == 4) {
                const uint4 x = *reinterpret_cast<const uint4*>(vt);
                o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w;
              } else if constexpr (Step::VD == 2) {
                const uint2 x = *reinterpret_cast<const uint2*>(vt);
                o[0] = x.x; o[1] = x.y;
              } else {
                o[0] = *reinterpret_cast<const uint32_t*>(vt);
              }
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) pk[ct] = softmax(ct, s[ct], k32, there32, look);
            values(st, pk, k32, there32, look);
          }
        }
      };
      go_through(std::false_type{});
      float all = 0.0f;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        f32x4 of_column = acc[ct][0];
#pragma unroll
        for (int i = 1; i < VW; ++i) of_column += acc[ct][i];
        all += live[ct] ? (of_column[0] + of_column[1]) + (of_column[2] + of_column[3]) : 0.0f;
      }
      const bool has_nan = __any(all != all);
      if (lane == 0) red[wave] = has_nan;       // all four wavefronts or none: they fetch for one another
      __syncthreads();
      if (scalar((uint32_t)(red[0] | red[1] | red[2] | red[3]))) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
          for (int i = 0; i < VW; ++i) acc[ct][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
          m[ct] = -INFINITY; l[ct] = Sum{};
        }
        go_through(std::true_type{});
      }
    } else {
      // ---- the keys, a step at a time, the next one's on their way meanwhile
      const int32_t round = (int32_t)D::unit(w);
      int32_t kb = k_first + (w.wide || w.quad ? 0 : (int32_t)(wave * 32u));
      if (kb < k_end) {
        Ids next = blocks(kb);
        Step one, two;
        load(one, kb, next);
        uint32_t in_one = present(next), in_two;
        next = blocks(kb + round);
        while (true) {
          load(two, kb + round, next);
          in_two = present(next);
          next = blocks(kb + 2 * round);
          work(one, kb, in_one);
          kb += round;
          if (kb >= k_end) break;
          load(one, kb + round, next);
          in_one = present(next);
          next = blocks(kb + 2 * round);
          work(two, kb, in_two);
          kb += round;
          if (kb >= k_end) break;
        }
      }
    }

    if constexpr (TILED) {
      if (pieces == 1) {                        // all of a column is in its lanes: VW features of a row of V^T tiles each
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if (!live[ct]) continue;
          const uint32_t f = first_col + ct * COLS + col;
          bf16_t* out = a.out + (uint64_t)(w.row0 + f / a.group) * a.ld_out + (uint64_t)(kh * a.group + f % a.group) * DH + 4u * g * VW;
          const float l1 = l[ct][0], inv = l1 == 0.0f ? 0.0f : (E4M3 && a.v_scale ? a.v_scale[kh] : 1.0f) / l1;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t o[VW / 2];
#pragma unroll
            for (int i = 0; i < VW / 2; ++i) o[i] = pack_bf16x2(acc[ct][2 * i][j] * inv, acc[ct][2 * i + 1][j] * inv);
            if constexpr (VW == 8) *reinterpret_cast<uint4*>(out + j * VW) = make_uint4(o[0], o[1], o[2], o[3]);
            else *reinterpret_cast<uint2*>(out + j * VW) = make_uint2(o[0], o[1]);
          }
        }
        continue;
      }
    }

    if (twice) {
      auto both = [](float x) { return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x128, 0xf, 0xf, false)); };      // row_ror:8
#pragma unroll
      for (int i = 0; i < VW; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[0][i][j] = both(acc[0][i][j]);
      if constexpr (!TILED) l[0] = both(l[0]);
      live[0] = col < n_cols;
    }

    // ---- the four wavefronts' sums together
    __syncthreads();                          // the last group's have been read
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float l1;
      if constexpr (TILED) {
        l1 = l[ct][0];
      } else {
        l1 = l[ct] + __shfl_xor(l[ct], 16, 64);
        l1 += __shfl_xor(l1, 32, 64);
      }
      const uint32_t c = wave * TC + ct * COLS + col;
      if (g == 0) { sum_m[c] = m[ct]; sum_l[c] = l1; }
      if (!live[ct]) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < VW; i += 4)
          *reinterpret_cast<f32x4*>(sum_acc + c * STRIDE + (4u * g + (uint32_t)j) * VW + (uint32_t)i) =
              f32x4{acc[ct][i][j], acc[ct][i + 1][j], acc[ct][i + 2][j], acc[ct][i + 3][j]};
    }
    __syncthreads();
    for (uint32_t u = tid; u < (w.quad ? WAVES * TC : n_group) * DV; u += THREADS) {
      const uint32_t c = u / DV, d = u % DV * 4u;
      Joined j;
      if (w.quad) {
        const uint32_t x = c / TC;
        if (c % TC >= n_group || kh0 + x >= a.kv_heads) continue;
        j.add(sum_m[c], sum_l[c], *reinterpret_cast<const f32x4*>(sum_acc + c * STRIDE + d));
        put(w.row0, group_col, kh0 + x, c % TC, d, j);
        continue;
      }
      if (TILED || w.wide) {
        j.add(sum_m[c], sum_l[c], *reinterpret_cast<const f32x4*>(sum_acc + c * STRIDE + d));
      } else {
#pragma unroll
        for (uint32_t x = 0; x < WAVES; ++x)
          j.add(sum_m[x * TC + c], sum_l[x * TC + c], *reinterpret_cast<const f32x4*>(sum_acc + (x * TC + c) * STRIDE + d));
      }
      if (pieces == 1) { put(w.row0, group_col, kh, c, d, j); continue; }
      float* to = part_of(2u * wg + (at_begin ? 0u : 1u)) + c * STRIDE;
      share_out(to + 4 + d, j.o[0], j.o[1]);
      share_out(to + 6 + d, j.o[2], j.o[3]);
      if (d == 0) share_out(to, j.m, j.l);
    }
    if (pieces > 1) {
      const Cut x = {w.row0, group_col, kh, n_group, wg_first, pieces, 2u * wg_first + (group_first - pad <= share * wg_first ? 0u : 1u)};
      if (at_begin) cut[0] = x; else cut[1] = x;
    }
  }

  // ---- the last piece of a group to be done adds them up
  if (cut[0].pieces + cut[1].pieces == 0) return;
  shared_out();
  __syncthreads();
  uint32_t* const arrived = (uint32_t*)red;
  if (tid < 2) {
    const uint32_t pieces = tid ? cut[1].pieces : cut[0].pieces, wg_first = tid ? cut[1].wg_first : cut[0].wg_first;
    bool last = false;
    if (pieces) {
      last = atomicAdd(counters + wg_first, 1u) + 1u == pieces;
      if (last) __hip_atomic_store(counters + wg_first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    arrived[tid] = last;
  }
  __syncthreads();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!arrived[which]) continue;
    const Cut& x = cut[which];
    const uint32_t lanes = x.n_cols * DV, teams = max(1u, THREADS / lanes), team = tid / lanes;      // of threads, each with its pieces
    for (uint32_t u = tid % lanes; u < lanes && team < teams; u += THREADS) {
      const uint32_t c = u / DV, d = u % DV * 4u;
      Joined j;
      // eight pieces' loads at a time: a trip to memory each
      for (uint32_t i = team; i < x.pieces; i += 8u * teams) {
        float2 ml[8], lo[8], hi[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
          const uint32_t p = min(i + k * teams, x.pieces - 1u);
          const float* from = part_of(p ? 2u * (x.wg_first + p) : x.first_place) + c * STRIDE;
          ml[k] = shared_in(from); lo[k] = shared_in(from + 4 + d); hi[k] = shared_in(from + 6 + d);
        }
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
          if (i + k * teams < x.pieces) j.add(ml[k].x, ml[k].y, f32x4{lo[k].x, lo[k].y, hi[k].x, hi[k].y});
      }
      if (teams == 1) { put(x.row0, x.group_col, x.kh, c, d, j); continue; }
      float* to = sum_acc + tid * 8u;
      *reinterpret_cast<f32x4*>(to) = j.o;
      to[4] = j.m; to[5] = j.l;
    }
    if (teams > 1) {
      __syncthreads();
      if (tid < lanes) {
        Joined j;
        for (uint32_t i = 0; i < teams; ++i) {
          const float* from = sum_acc + (i * lanes + tid) * 8u;
          j.add(from[4], from[5], *reinterpret_cast<const f32x4*>(from));
        }
        put(x.row0, x.group_col, x.kh, tid / DV, tid % DV * 4u, j);
      }
      __syncthreads();
    }
  }
}

// Tiles of 16 columns a wavefront: heads of 64 have the registers for two, which sequences with many columns take.
constexpr uint32_t many_tiles(uint32_t dh) { return dh == 64 ? 2u : 1u; }
// Whether the keys go through the LDS.
bool tiled(uint32_t rows, uint32_t n_seq, uint32_t q_heads, uint32_t group, uint32_t dh) {
  const uint64_t groups = (uint64_t)rows * q_heads / TILED_GROUP;
  return (uint64_t)rows * group >= (uint64_t)TILED_COLS * n_seq && groups > (dh == 64 ? MAX_WGS - 1 : MAX_WGS / 4);
}
// Columns that a piece may have.
uint32_t part_columns(uint32_t rows, uint32_t n_seq, uint32_t q_heads, uint32_t group, uint32_t dh) {
  return (uint32_t)std::min<uint64_t>(tiled(rows, n_seq, q_heads, group, dh) ? TILED_GROUP : COLS * WAVES * many_tiles(dh), (uint64_t)rows * group);
}

template <int DH, bool E4M3, int CT, bool TILED>
hipError_t launch_paged(const PagedArgs& a, uint32_t rows, void* scratch, hipStream_t st) {
  constexpr uint32_t TC = COLS * CT, GC = TILED ? TILED_GROUP : TC;
  uint32_t* counters = (uint32_t*)scratch;
  float* parts = (float*)scratch + MAX_WGS;
  // units that there can be: column tiles, key heads, the longest sequence that the tables have room for
  const uint64_t groups = (((uint64_t)rows * a.group + GC - 1) / GC + a.n_seq) * a.kv_heads;
  const uint64_t units = (((uint64_t)a.max_blocks << a.block_shift) + 31) / 32;
  const bool few = a.n_seq <= 64 && (double)groups * (double)(2 * units + 2) < 4e9;      // 32 bits hold the sums, padding included
  const uint32_t sums = WAVES * TC * (DH + 4) * 4 + WAVES * TC * 8, row = DH * (E4M3 ? 1u : 2u), tiles = TILED ? 8u * tile_step(row) * row : 0u;
  const uint32_t fixed = std::max(sums, tiles) + WAVES * 8, lds = fixed + (few ? 0 : a.n_seq * 8);
  if (lds > 60u * 1024) {                       // the limit that all calls have in common: another thread's call finds it no lower than its own
    hipError_t e = hipFuncSetAttribute((const void*)paged_attention_kernel<DH, E4M3, CT, TILED>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)(fixed + CACHE_MAX_SEQ * 8));
    if (e != hipSuccess) return e;
  }
  const uint32_t wgs = (uint32_t)std::min<uint64_t>(MAX_WGS, (groups * ((units + MIN_PIECE - 1) / MIN_PIECE) + 7) / 8 * 8);
  const bool may_be_wide = !TILED && rows * a.group > 2 * TC && (a.starts || a.group > 2 * TC);
  paged_attention_kernel<DH, E4M3, CT, TILED><<<wgs, THREADS, lds, st>>>(a, counters, parts, part_columns(rows, a.n_seq, a.q_heads, a.group, DH), few, may_be_wide);
  return hipGetLastError();
}

template <int DH, bool E4M3>
hipError_t launch_paged(const PagedArgs& a, void* scratch, hipStream_t st) {
  const uint32_t rows = a.starts ? a.n_rows : std::min(a.n_rows, a.n_seq);
  if (rows == 0) return hipSuccess;
  if (tiled(rows, a.n_seq, a.q_heads, a.group, DH)) return launch_paged<DH, E4M3, 2, true>(a, rows, scratch, st);
  if constexpr (many_tiles(DH) > 1)
    if ((uint64_t)rows * a.group >= (uint64_t)MANY_COLS * a.n_seq) return launch_paged<DH, E4M3, (int)many_tiles(DH), false>(a, rows, scratch, st);
  return launch_paged<DH, E4M3, 1, false>(a, rows, scratch, st);
}

}  // namespace

uint64_t paged_attention_scratch(uint32_t n_rows, uint32_t n_seq, uint32_t q_heads, uint32_t head_dim) {
  return MAX_WGS * 4 + 2ull * MAX_WGS * part_columns(n_rows, n_seq, q_heads, q_heads, head_dim) * (head_dim + 4) * 4;
}

hipError_t launch_paged_attention(const PagedArgs& a, uint32_t head_dim, bool e4m3, void* scratch, hipStream_t st) {
  if (head_dim == 128) return e4m3 ? launch_paged<128, true>(a, scratch, st) : launch_paged<128, false>(a, scratch, st);
  return e4m3 ? launch_paged<64, true>(a, scratch, st) : launch_paged<64, false>(a, scratch, st);
}

__global__ __launch_bounds__(256) void last_rows_kernel(const uint4* __restrict__ x, const int32_t* __restrict__ starts, uint32_t n_rows,
                                                        uint32_t chunks, uint4* __restrict__ out) {
  const int32_t first = starts[blockIdx.x], end = starts[blockIdx.x + 1];
  const bool some = end > first && first >= 0 && (uint32_t)end <= n_rows;
  for (uint32_t c = threadIdx.x; c < chunks; c += 256)
    out[(uint64_t)blockIdx.x * chunks + c] = some ? x[(uint64_t)(end - 1) * chunks + c] : make_uint4(0u, 0u, 0u, 0u);
}
hipError_t launch_last_rows(const void* x, const int32_t* starts, uint32_t n_rows, uint32_t n_seq, uint32_t d, void* out, hipStream_t st) {
  last_rows_kernel<<<n_seq, 256, 0, st>>>((const uint4*)x, starts, n_rows, d / 8, (uint4*)out);
  return hipGetLastError();
}

}  // namespace qzo
