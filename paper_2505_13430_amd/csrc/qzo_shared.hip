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

// A row's head a team of DH / 4 lanes.
template <int DH>
__global__ __launch_bounds__(256) void join_shares_kernel(SharedArgs a, bool e4m3) {
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
  j.add(head_own[0], head_own[1], o_own);
  const float inv = (e4m3 && a.v_scale ? a.v_scale[head / a.group] : 1.0f) / j.l;
  bf16_t* const to = a.out + (uint64_t)row * a.ld_out + (uint64_t)head * DH + d;
  *reinterpret_cast<uint2*>(to) = j.l == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(j.o[0] * inv, j.o[1] * inv), pack_bf16x2(j.o[2] * inv, j.o[3] * inv));
}

uint32_t shared_part_columns(uint32_t n_rows, uint32_t group) {
  return (uint32_t)std::min<uint64_t>(TILED_GROUP, (uint64_t)n_rows * group);
}
uint64_t parts_bytes(uint32_t n_rows, uint32_t group, uint32_t head_dim) {
  return 2ull * MAX_WGS * shared_part_columns(n_rows, group) * (head_dim + 4) * 4;
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
  const uint32_t fixed = std::max(sums, tiles) + WAVES * 8, lds = fixed + (few ? 0 : n_items * 8) + (2 * a.n_groups + 1) * 4;
  if (lds > 60u * 1024) {                       // the limit that all calls have in common
    hipError_t e = hipFuncSetAttribute((const void*)paged_attention_kernel<DH, E4M3, CT, TILED, true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)(fixed + CACHE_MAX_SEQ * 8 + (2 * SHARED_MAX_GROUPS + 1) * 4));
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
  hipError_t e;
  if (of_group >= TILED_COLS || a.n_groups + a.n_seq > CACHE_MAX_SEQ) {
    e = launch_by_columns<DH, E4M3>(a, rows, of_group, 0, a.n_groups, scratch, st);
    if (e == hipSuccess) e = launch_by_columns<DH, E4M3>(a, rows, of_seq, a.n_groups, a.n_seq, scratch, st);
  } else {
    e = launch_by_columns<DH, E4M3>(a, rows, of_group, 0, a.n_groups + a.n_seq, scratch, st);
  }
  if (e != hipSuccess) return e;
  const uint64_t pairs = (uint64_t)a.n_rows * a.q_heads, per = 1024 / DH;
  join_shares_kernel<DH><<<(uint32_t)((pairs + per - 1) / per), 256, 0, st>>>(a, E4M3);
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
