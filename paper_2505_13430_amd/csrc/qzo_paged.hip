// Attention of the newest tokens of sequences over a paged cache: launches of the kernel in qzo_paged_kernel.hpp.
#include "qzo_paged_kernel.hpp"

namespace qzo {
namespace {

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
    hipError_t e = hipFuncSetAttribute((const void*)paged_attention_kernel<DH, E4M3, CT, TILED, false>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)(fixed + CACHE_MAX_SEQ * 8));
    if (e != hipSuccess) return e;
  }
  const uint32_t wgs = (uint32_t)std::min<uint64_t>(MAX_WGS, (groups * ((units + MIN_PIECE - 1) / MIN_PIECE) + 7) / 8 * 8);
  const bool may_be_wide = !TILED && rows * a.group > 2 * TC && (a.starts || a.group > 2 * TC);
  paged_attention_kernel<DH, E4M3, CT, TILED, false><<<wgs, THREADS, lds, st>>>(a, counters, parts, part_columns(rows, a.n_seq, a.q_heads, a.group, DH), few, may_be_wide);
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
