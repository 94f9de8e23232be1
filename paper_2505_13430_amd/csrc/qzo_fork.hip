// Sequences of the paged cache that fork: tables that share blocks, blocks given back and copied, a pool made compact.
#include <algorithm>
#include "qzo_device.hpp"
#include "qzo_kernels.hpp"

namespace qzo {
namespace {

constexpr uint32_t THREADS = 256, WAVES = THREADS / 64;

// Inclusive sum over a workgroup's threads; total: of all of them.  N: its wavefronts; red: [N], read before the next call by way of its first barrier.
template <uint32_t N = WAVES>
__device__ __forceinline__ uint32_t group_scan(uint32_t v, uint32_t* total, uint32_t* red) {
  const uint32_t upto = lane_scan(v);
  __syncthreads();
  if ((threadIdx.x & 63u) == 63u) red[threadIdx.x >> 6] = upto;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < N; ++w) {
    if (w < (threadIdx.x >> 6)) before += red[w];
    all += red[w];
  }
  *total = all;
  return before + upto;
}

__device__ __forceinline__ uint32_t blocks_of(int32_t length, const ForkArgs& a) {       // of a length that the tables have room for
  const uint32_t room = a.max_blocks << a.block_shift;
  return (min((uint32_t)max(length, 0), room) + (1u << a.block_shift) - 1u) >> a.block_shift;
}

// ------------------------------------------------------------------ fork ----
// A sequence of before lives on if it is any sequence's parent.  A block is free again if it was held, and by none that lives on.
// Every held block gets a mark, the highest of its holders': n_seq + 1 of one that lives on, n_seq - i of sequence i that does
// not.  So the mark tells which blocks are free, and which of several holders gives one back.
//   1. mark: the tables are put aside (they are rewritten in place), the marks made; a workgroup of its own finds who takes a block for a copy.
//   2. count: how many blocks each sequence gives back; the last workgroup to be done has all the counts and adds them up.
//   3. write: tables, lengths, the stack, copies; the marks go back to zero.
// Whole numbers and maxima: the order of the atomics changes nothing.
// 128 x 6 sequences of up to 253 blocks: 21 us, of which 5, 11 and 6 are the three launches'; latency is what they consist of (the bytes take 0.2 us).
__global__ __launch_bounds__(THREADS) void fork_mark_kernel(ForkArgs a) {
  const uint32_t i = blockIdx.x, tid = threadIdx.x;
  extern __shared__ int32_t first_child[];            // [n_seq], of the last workgroup
  __shared__ uint32_t lives, flags, red[WAVES];
  if (i == a.n_seq) {
    // ---- beside the marks: which copy is a sequence's, what is wrong
    for (uint32_t j = tid; j < a.n_seq; j += THREADS) first_child[j] = (int32_t)a.n_seq;
    if (tid == 0) flags = 0;
    __syncthreads();
    const int64_t room = (int64_t)a.max_blocks << a.block_shift;
    uint32_t wrong = 0;
#pragma unroll 4
    for (uint32_t j = tid; j < a.n_seq; j += THREADS) {
      const int32_t p = a.parents[j], length = a.lengths[j];
      if (p >= (int32_t)a.n_seq || length < 0) wrong |= 1u;
      if (length > room) wrong |= 2u;
      if (p >= 0 && p < (int32_t)a.n_seq) atomicMin(first_child + p, (int32_t)j);
    }
    if (wrong) atomicOr(&flags, wrong);
    __syncthreads();
    const uint32_t per = (a.n_seq + THREADS - 1) / THREADS, first = min(tid * per, a.n_seq), end = min(first + per, a.n_seq);
    auto copies = [&](uint32_t j) {
      const int32_t p = a.parents[j];
      const bool known = p >= 0 && p < (int32_t)a.n_seq;
      return known && (a.lengths[known ? p : 0] & ((1 << a.block_shift) - 1)) && first_child[known ? p : 0] != (int32_t)j;
    };
    uint32_t n_copy, copy = 0;
#pragma unroll 4
    for (uint32_t j = first; j < end; ++j) copy += copies(j);
    copy = group_scan(copy, &n_copy, red) - copy;
#pragma unroll 4
    for (uint32_t j = first; j < end; ++j) {
      const bool one = copies(j);
      a.copy_of[j] = one ? (int32_t)copy : -1;
      if (one) a.taker[copy] = (int32_t)j;
      copy += one;
    }
    if (tid == 0) *a.plan = ForkPlan{a.state->n_free, 0, (int32_t)n_copy, (int32_t)flags};
    return;
  }
  if (tid == 0) lives = 0;
  const int32_t length = a.lengths[i];
  const int32_t* const row = a.tables + (uint64_t)i * a.max_blocks;
  int32_t* const aside = a.aside + (uint64_t)i * a.max_blocks;
  const int32_t id0 = row[min(tid, a.max_blocks - 1u)];          // on its way beside the parents
  __syncthreads();
  bool found = false;
#pragma unroll 4
  for (uint32_t j = tid; j < a.n_seq; j += THREADS) found |= a.parents[j] == (int32_t)i;
  if (__any(found) && (tid & 63u) == 0) lives = 1;
  __syncthreads();
  if (tid == 0) a.old_lengths[i] = length;
  const uint32_t mark = lives ? a.n_seq + 1u : a.n_seq - i, n = blocks_of(length, a);
  for (uint32_t j = tid; j < n; j += THREADS) {
    const int32_t id = j == tid ? id0 : row[j];
    aside[j] = id;
    if ((uint32_t)id < a.n_blocks) atomicMax(a.marks + id, mark);
  }
}

constexpr uint32_t COUNT_WGS = 128;
__global__ __launch_bounds__(THREADS) void fork_count_kernel(ForkArgs a) {
  const uint32_t tid = threadIdx.x, lane = tid & 63u;
  __shared__ uint32_t red[WAVES], last;
  const ForkPlan plan = *a.plan;                     // of the last workgroup's use
  // a wavefront a sequence; few workgroups, for all count at one place, 10 ns each (768 sequences with a workgroup each 14.4 us)
  for (uint32_t i = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * WAVES + (tid >> 6))); i < a.n_seq; i += COUNT_WGS * WAVES) {
    const int32_t* const aside = a.aside + (uint64_t)i * a.max_blocks;
    const uint32_t n = blocks_of(a.old_lengths[i], a);
    uint32_t count = 0;
#pragma unroll 4
    for (uint32_t j = lane; j < n; j += 64) {
      const int32_t id = aside[j];
      count += (uint32_t)id < a.n_blocks && a.marks[(uint32_t)id < a.n_blocks ? id : 0] == a.n_seq - i;
    }
    count = (uint32_t)__builtin_amdgcn_readlane((int)lane_scan(count), 63);
    if (lane == 0) __hip_atomic_store(a.given + i, count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) last = atomicAdd(a.arrived, 1u) + 1u == gridDim.x;
  __syncthreads();
  if (!last) return;
  if (tid == 0) __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // ---- what the sequences before give back, a few sequences a thread
  constexpr uint32_t PER = CACHE_MAX_SEQ / THREADS;
  const uint32_t per = (a.n_seq + THREADS - 1) / THREADS, j_first = tid * per;
  uint32_t given[PER], back = 0, n_back;
#pragma unroll
  for (uint32_t x = 0; x < PER; ++x) {
    if (x >= per) break;
    given[x] = __hip_atomic_load(a.given + min(j_first + x, a.n_seq - 1u), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
#pragma unroll
  for (uint32_t x = 0; x < PER; ++x)
    if (x < per && j_first + x < a.n_seq) back += given[x];
  back = group_scan(back, &n_back, red) - back;
#pragma unroll
  for (uint32_t x = 0; x < PER; ++x)
    if (x < per && j_first + x < a.n_seq) { a.before[j_first + x] = back; back += given[x]; }
  const int32_t n_free = plan.n_free, n_copy = plan.n_copy, flags = plan.status;
  int32_t status = QZO_OK;
  if ((flags & 1) || n_free < 0 || (uint32_t)n_free > a.n_blocks) status = QZO_ERR_ARG;
  else if (flags & 2) status = QZO_ERR_SHAPE;
  else if ((uint64_t)n_free + n_back > a.n_blocks) status = QZO_ERR_ARG;
  else if ((uint32_t)n_copy > (uint32_t)n_free + n_back) status = QZO_ERR_WORKSPACE;
  if (tid == 0) {
    const bool ok = status == QZO_OK;
    *a.plan = ForkPlan{n_free, ok ? (int32_t)n_back : 0, ok ? n_copy : 0, status};
    *a.state = qzo_cache_state{ok ? n_free + (int32_t)n_back - n_copy : n_free, 0, status, ok ? n_copy : 0};
  }
}

__global__ __launch_bounds__(THREADS) void fork_write_kernel(ForkArgs a) {
  const uint32_t tid = threadIdx.x;
  const ForkPlan plan = *a.plan;
  const bool ok = plan.status == QZO_OK;
  const uint32_t shift = a.block_shift;
  auto aside_of = [&](uint32_t s) { return a.aside + (uint64_t)s * a.max_blocks; };
  if (blockIdx.x >= a.n_seq) {          // a group: how many of the blocks at the head are the same for all its sequences that live
    const uint32_t g = blockIdx.x - a.n_seq;
    const uint32_t s0 = (uint32_t)min(max(a.group_starts[g], 0), (int32_t)a.n_seq), s1 = max(s0, (uint32_t)min(max(a.group_starts[g + 1], 0), (int32_t)a.n_seq));
    __shared__ uint32_t lead, same;
    if (tid == 0) { lead = ~0u; same = ~0u; }
    __syncthreads();
    // (lengths may have been rewritten by now: those of before are aside)
    auto full = [&](uint32_t s, uint32_t* from) -> uint32_t {
      const int32_t p = ok ? a.parents[s] : (int32_t)s;
      *from = (uint32_t)max(p, 0);
      return p < 0 ? 0u : (uint32_t)min(max(a.old_lengths[p], 0), (int32_t)(a.max_blocks << shift));
    };
    uint32_t from;
    for (uint32_t s = s0 + tid; s < s1; s += THREADS)
      if (full(s, &from)) { atomicMin(&lead, s); break; }
    __syncthreads();
    if (lead != ~0u) {
      uint32_t of_lead;
      const uint32_t n_lead = full(lead, &of_lead) >> shift;
      const int32_t* const x = aside_of(of_lead);
      for (uint32_t s = s0; s < s1; ++s) {
        const uint32_t length = full(s, &from);
        if (!length) continue;
        const uint32_t n = min(length >> shift, n_lead);
        const int32_t* const y = aside_of(from);
        if (tid == 0) atomicMin(&same, n);
        if (from == of_lead) continue;
        for (uint32_t j = tid; j < n; j += THREADS)
          if (x[j] != y[j]) { atomicMin(&same, j); break; }
      }
    }
    __syncthreads();
    if (tid == 0) a.shared[g] = lead == ~0u ? 0 : (int32_t)(same << shift);
    return;
  }
  const uint32_t i = blockIdx.x;
  __shared__ uint32_t red[WAVES];
  // ---- what old sequence i gives back: block number r of all is at n_free + r of the stack, or is taken by copy n_back - 1 - r
  const uint32_t n_old = blocks_of(a.old_lengths[i], a);
  const int32_t* const old = aside_of(i);
  const uint32_t mine = a.n_seq - i;
  const int32_t kept = plan.n_back - min(plan.n_back, plan.n_copy);           // of those given back that stay on the stack
  uint32_t r0 = a.before[i];
  for (uint32_t j0 = 0; j0 < n_old; j0 += THREADS) {
    const uint32_t j = j0 + tid;
    const int32_t id = j < n_old ? old[j] : -1;
    const uint32_t mark = (uint32_t)id < a.n_blocks ? a.marks[id] : 0u;
    uint32_t all;
    const uint32_t r = r0 + group_scan(mark == mine, &all, red) - 1u;
    r0 += all;
    // who has the highest mark takes it away: nobody else's comparison above comes out another way
    if (mark == mine || mark > a.n_seq) a.marks[id] = 0;
    if (mark != mine || !ok) continue;
    if ((int32_t)r < kept) {
      a.free[plan.n_free + (int32_t)r] = id;
    } else {
      const int32_t k = plan.n_back - 1 - (int32_t)r, s = a.taker[k];
      const int32_t length = a.old_lengths[a.parents[s]];
      a.tables[(uint64_t)s * a.max_blocks + (uint32_t)(length >> shift)] = id;
      a.copies[k].to = id;
    }
  }
  // ---- new sequence i
  if (!ok) return;
  const int32_t p = a.parents[i], length = p < 0 ? 0 : a.old_lengths[p], k = a.copy_of[i];
  if (tid == 0) a.lengths[i] = length;
  if (p < 0) return;
  const uint32_t n = (uint32_t)(length + (1 << shift) - 1) >> shift;
  const int32_t* const from = aside_of((uint32_t)p);
  int32_t* const to = a.tables + (uint64_t)i * a.max_blocks;
  if (p != (int32_t)i)
    for (uint32_t j = tid; j < (k < 0 ? n : n - 1u); j += THREADS) to[j] = from[j];
  if (k >= 0 && tid == 0) {
    a.copies[k].from = from[n - 1u];
    a.copies[k].tokens = length & ((1 << shift) - 1);
    a.copies[k].reserved = 0;
    if (k >= plan.n_back) {             // one that was on the stack before
      const int32_t id = a.free[plan.n_free - 1 - (k - plan.n_back)];
      a.copies[k].to = id;
      to[n - 1u] = id;
    }
  }
}

// The same with few sequences and a small pool, in one workgroup: tables and marks in the LDS.  Latency is all there is to it: 8 beams behind 2500
// tokens 8.6 us, in three launches 13.8.
constexpr uint32_t SMALL_THREADS = 1024, SMALL_SEQ = 256, SMALL_ENTRIES = 16384, SMALL_BLOCKS = 16384;
__global__ __launch_bounds__(SMALL_THREADS) void fork_small_kernel(ForkArgs a) {
  extern __shared__ int32_t small_lds[];
  int32_t* const aside = small_lds;                                       // [n_seq, max_blocks]
  uint32_t* const marks = (uint32_t*)(aside + a.n_seq * a.max_blocks);    // [n_blocks]
  __shared__ int32_t length[SMALL_SEQ], parent[SMALL_SEQ], first_child[SMALL_SEQ], copy_of[SMALL_SEQ], taker[SMALL_SEQ];
  __shared__ uint32_t given[SMALL_SEQ], red[SMALL_THREADS / 64], flags;
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, shift = a.block_shift, mask = (1u << shift) - 1u;
  const uint32_t WAVES16 = SMALL_THREADS / 64;
  const int64_t room = (int64_t)a.max_blocks << shift;
  const int32_t n_free = a.state->n_free;
  if (tid == 0) flags = 0;
  if (tid < a.n_seq) { length[tid] = a.lengths[tid]; parent[tid] = a.parents[tid]; first_child[tid] = (int32_t)a.n_seq; given[tid] = 0; }
  for (uint32_t e = tid; e < a.n_seq * a.max_blocks; e += SMALL_THREADS) aside[e] = a.tables[e];
  for (uint32_t b = tid; b < a.n_blocks; b += SMALL_THREADS) marks[b] = 0;
  __syncthreads();
  if (tid < a.n_seq) {
    const int32_t p = parent[tid], l = length[tid];
    const uint32_t wrong = (p >= (int32_t)a.n_seq || l < 0 ? 1u : 0u) | (l > room ? 2u : 0u);
    if (wrong) atomicOr(&flags, wrong);
    if (p >= 0 && p < (int32_t)a.n_seq) atomicMin(first_child + p, (int32_t)tid);
  }
  __syncthreads();
  // a wavefront a sequence
  for (uint32_t i = wave; i < a.n_seq; i += WAVES16) {
    const uint32_t mark = first_child[i] < (int32_t)a.n_seq ? a.n_seq + 1u : a.n_seq - i, n = blocks_of(length[i], a);
    for (uint32_t j = lane; j < n; j += 64) {
      const int32_t id = aside[i * a.max_blocks + j];
      if ((uint32_t)id < a.n_blocks) atomicMax(marks + id, mark);
    }
  }
  __syncthreads();
  auto mine = [&](uint32_t i, uint32_t j, uint32_t n) {
    const int32_t id = j < n ? aside[i * a.max_blocks + j] : -1;
    return (uint32_t)id < a.n_blocks && marks[id] == a.n_seq - i;
  };
  for (uint32_t i = wave; i < a.n_seq; i += WAVES16) {
    if (first_child[i] < (int32_t)a.n_seq) continue;
    const uint32_t n = blocks_of(length[i], a);
    uint32_t count = 0;
    for (uint32_t j0 = 0; j0 < n; j0 += 64) count += (uint32_t)__popcll(__ballot(mine(i, j0 + lane, n)));
    if (lane == 0) given[i] = count;
  }
  __syncthreads();
  const uint32_t back = tid < a.n_seq ? given[tid] : 0u;
  const int32_t p0 = tid < a.n_seq ? parent[tid] : -1;
  const uint32_t copy = p0 >= 0 && p0 < (int32_t)a.n_seq && ((uint32_t)length[p0] & mask) && first_child[p0] != (int32_t)tid;
  uint32_t n_back, n_copy;
  const uint32_t back_before = group_scan<SMALL_THREADS / 64>(back, &n_back, red) - back;
  const uint32_t copy_before = group_scan<SMALL_THREADS / 64>(copy, &n_copy, red) - copy;
  int32_t status = QZO_OK;
  if ((flags & 1u) || n_free < 0 || (uint32_t)n_free > a.n_blocks) status = QZO_ERR_ARG;
  else if (flags & 2u) status = QZO_ERR_SHAPE;
  else if ((uint64_t)n_free + n_back > a.n_blocks) status = QZO_ERR_ARG;
  else if (n_copy > (uint32_t)n_free + n_back) status = QZO_ERR_WORKSPACE;
  const bool ok = status == QZO_OK;
  if (tid < a.n_seq) {
    given[tid] = back_before;
    copy_of[tid] = copy ? (int32_t)copy_before : -1;
    if (copy) taker[copy_before] = (int32_t)tid;
    if (ok) a.lengths[tid] = p0 < 0 ? 0 : length[p0];
  }
  if (tid == 0) *a.state = qzo_cache_state{ok ? n_free + (int32_t)n_back - (int32_t)n_copy : n_free, 0, status, ok ? (int32_t)n_copy : 0};
  __syncthreads();
  const int32_t kept = (int32_t)n_back - (int32_t)min(n_back, n_copy);
  for (uint32_t i = wave; ok && i < a.n_seq; i += WAVES16) {
    if (first_child[i] >= (int32_t)a.n_seq) {              // gives back
      const uint32_t n = blocks_of(length[i], a);
      int32_t r0 = (int32_t)given[i];
      for (uint32_t j0 = 0; j0 < n; j0 += 64) {
        const bool is = mine(i, j0 + lane, n);
        const uint64_t who = __ballot(is);
        const int32_t r = r0 + (int32_t)__popcll(who & ((1ull << lane) - 1ull));
        r0 += (int32_t)__popcll(who);
        if (!is) continue;
        const int32_t id = aside[i * a.max_blocks + j0 + lane];
        if (r < kept) {
          a.free[n_free + r] = id;
        } else {
          const int32_t k = (int32_t)n_back - 1 - r, s = taker[k];
          a.tables[(uint64_t)s * a.max_blocks + ((uint32_t)length[parent[s]] >> shift)] = id;
          a.copies[k].to = id;
        }
      }
    }
    const int32_t p = parent[i], k = copy_of[i];
    if (p < 0) continue;
    const uint32_t n = ((uint32_t)length[p] + mask) >> shift;
    if (p != (int32_t)i)
      for (uint32_t j = lane; j < (k < 0 ? n : n - 1u); j += 64) a.tables[(uint64_t)i * a.max_blocks + j] = aside[(uint32_t)p * a.max_blocks + j];
    if (k >= 0 && lane == 0) {
      a.copies[k].from = aside[(uint32_t)p * a.max_blocks + n - 1u];
      a.copies[k].tokens = (int32_t)((uint32_t)length[p] & mask);
      a.copies[k].reserved = 0;
      if (k >= (int32_t)n_back) {
        const int32_t id = a.free[n_free - 1 - (k - (int32_t)n_back)];
        a.copies[k].to = id;
        a.tables[(uint64_t)i * a.max_blocks + n - 1u] = id;
      }
    }
  }
  // groups: a wavefront each
  for (uint32_t g = wave; g < a.n_groups; g += WAVES16) {
    const uint32_t s0 = (uint32_t)min(max(a.group_starts[g], 0), (int32_t)a.n_seq), s1 = max(s0, (uint32_t)min(max(a.group_starts[g + 1], 0), (int32_t)a.n_seq));
    uint32_t lead = ~0u, same = ~0u;
    for (uint32_t s = s0; s < s1; ++s) {
      const int32_t p = ok ? parent[s] : (int32_t)s;
      const uint32_t l = p < 0 ? 0u : (uint32_t)min((int64_t)max(length[p], 0), room);
      if (!l) continue;
      const uint32_t n = l >> shift;
      if (lead == ~0u) { lead = (uint32_t)p; same = n; continue; }
      same = min(same, n);
      for (uint32_t j0 = 0; lead != (uint32_t)p && j0 < same; j0 += 64) {
        const uint32_t j = j0 + lane;
        const uint64_t other = __ballot(j < same && aside[lead * a.max_blocks + j] != aside[(uint32_t)p * a.max_blocks + j]);
        if (other) { same = j0 + (uint32_t)__builtin_ctzll(other); break; }
      }
    }
    if (lane == 0) a.shared[g] = lead == ~0u ? 0 : (int32_t)(same << shift);
  }
}

// ------------------------------------------------------------------ compact ----
// Held blocks are marked; n of them: those from n on go to the places below n that none holds, in order.
// Four launches that wait for one another, 2.7 + 4.7 + 4.2 + 2.9 us for 1400 blocks, 3.1 + 6.1 + 6.8 + 4.3 for 150001 (in a graph 13 and 19 us): each step
// needs all of the one before.
constexpr uint32_t CHUNK = 8 * THREADS;           // blocks that a workgroup counts
__global__ __launch_bounds__(THREADS) void compact_mark_kernel(ForkArgs a) {
  const uint32_t i = blockIdx.x, n = blocks_of(a.lengths[i], a);
  const int32_t* const row = a.tables + (uint64_t)i * a.max_blocks;
  for (uint32_t j = threadIdx.x; j < n; j += THREADS)
    if ((uint32_t)row[j] < a.n_blocks) a.marks[row[j]] = 1u;
}
__global__ __launch_bounds__(THREADS) void compact_count_kernel(ForkArgs a) {
  const uint32_t tid = threadIdx.x, b0 = blockIdx.x * CHUNK + tid * 8u;
  __shared__ uint32_t red[WAVES], last;
  uint32_t count = 0, all;
#pragma unroll
  for (uint32_t x = 0; x < 8; ++x) count += b0 + x < a.n_blocks && a.marks[b0 + x];
  group_scan(count, &all, red);
  if (tid == 0) {
    __hip_atomic_store(a.given + blockIdx.x, all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = atomicAdd(a.arrived, 1u) + 1u == gridDim.x;
  }
  __syncthreads();
  if (!last) return;
  if (tid == 0) __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  uint32_t held = 0;
  for (uint32_t c0 = 0; c0 < gridDim.x; c0 += THREADS) {
    const uint32_t c = c0 + tid, n = c < gridDim.x ? __hip_atomic_load(a.given + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
    const uint32_t upto = group_scan(n, &all, red);
    if (c < gridDim.x) a.given[c] = held + upto - n;
    held += all;
  }
  // held blocks before the first of the others' places: the chunk that n_held falls into is counted once more
  const uint32_t chunk = min(held / CHUNK, gridDim.x - 1u);
  __syncthreads();
  count = 0;
#pragma unroll
  for (uint32_t x = 0; x < 8; ++x) {
    const uint32_t b = chunk * CHUNK + tid * 8u + x;
    count += b < held && b < a.n_blocks && a.marks[b];
  }
  group_scan(count, &all, red);
  if (tid == 0) {
    const uint32_t near = a.given[chunk] + all;
    *a.plan = ForkPlan{(int32_t)held, (int32_t)near, 0, QZO_OK};
    *a.state = qzo_cache_state{(int32_t)(a.n_blocks - held), 0, QZO_OK, (int32_t)(held - near)};
  }
}
// Where each block goes: the i-th of the far ones keeps i + 1 in its mark until the tables have been rewritten, the others 0.
__global__ __launch_bounds__(THREADS) void compact_place_kernel(ForkArgs a) {
  const uint32_t tid = threadIdx.x, b0 = blockIdx.x * CHUNK + tid * 8u;
  __shared__ uint32_t red[WAVES];
  const uint32_t held = (uint32_t)a.plan->n_free, near = (uint32_t)a.plan->n_back;
  uint32_t is[8], count = 0, all;
#pragma unroll
  for (uint32_t x = 0; x < 8; ++x) {
    is[x] = b0 + x < a.n_blocks && a.marks[b0 + x];
    count += is[x];
  }
  uint32_t before = a.given[blockIdx.x] + group_scan(count, &all, red) - count;
#pragma unroll
  for (uint32_t x = 0; x < 8; ++x) {
    const uint32_t b = b0 + x;
    if (b >= a.n_blocks) break;
    if (is[x] && b >= held) a.copies[before - near].from = (int32_t)b;
    if (!is[x] && b < held) a.copies[b - before].to = (int32_t)b;
    a.place[b] = is[x] && b >= held ? before - near : ~0u;
    a.marks[b] = 0;
    before += is[x];
    if (b < a.n_blocks - held) a.free[b] = (int32_t)(a.n_blocks - 1u - b);
  }
}
__global__ __launch_bounds__(THREADS) void compact_write_kernel(ForkArgs a) {
  const uint32_t tid = threadIdx.x;
  if (blockIdx.x < a.n_seq) {
    const uint32_t i = blockIdx.x, n = blocks_of(a.lengths[i], a);
    for (uint32_t j = tid; j < n; j += THREADS) {
      const uint64_t at = (uint64_t)i * a.max_blocks + j;
      int32_t id = a.tables[at];
      if ((uint32_t)id < a.n_blocks) {
        const uint32_t r = a.place[id];
        if (r != ~0u) id = a.copies[r].to;
      }
      a.new_tables[at] = id;
    }
    return;
  }
  const uint32_t moved = (uint32_t)a.state->n_taken;
  for (uint32_t r = (blockIdx.x - a.n_seq) * THREADS + tid; r < moved; r += (gridDim.x - a.n_seq) * THREADS) {
    a.copies[r].tokens = 1 << a.block_shift;
    a.copies[r].reserved = 0;
  }
}

// ------------------------------------------------------------------ copies ----
// The first tokens of a block are consecutive for each layer, pool and head: such a run is a wavefront's, 16 bytes a lane, four times
// on their way.  A row of the grid takes every gridDim.y-th entry.  Bound by memory: 700 e4m3 blocks of 8 layers, 0.73 GB, 298 us, 4.9 TB/s read and
// written, which is a large copy's rate; three blocks, 25 MB, 5.0 us.  (The four pieces in variables of their own: as an array they go to the LDS, by an
// index for which every workgroup reads its launch packet in host memory: 18 us in place of 5.)
__global__ __launch_bounds__(THREADS) void copy_blocks_kernel(CopyArgs a) {
  const uint32_t lane = threadIdx.x & 63u;
  const uint32_t run = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * WAVES + (threadIdx.x >> 6))), runs = a.layers * 2u * a.kv_heads;
  const uint32_t n = a.count ? (uint32_t)min(max(*a.count, 0), (int32_t)a.n_copies) : a.n_copies;
  if (run >= runs) return;
  const uint32_t pool = run / a.kv_heads, head = run - pool * a.kv_heads;             // layer by layer, k and v
  const uint64_t run_bytes = (uint64_t)a.row_bytes << a.block_shift;
  unsigned char* const base = (unsigned char*)(pool & 1u ? a.v : a.k) + ((uint64_t)(pool >> 1) * a.n_blocks * a.kv_heads + head) * run_bytes;
  const uint64_t block_bytes = run_bytes * a.kv_heads;
  for (uint32_t e = blockIdx.y; e < n; e += gridDim.y) {
    const qzo_block_copy c = a.copies[e];
    if ((uint32_t)c.from >= a.n_blocks || (uint32_t)c.to >= a.n_blocks || c.from == c.to || c.tokens <= 0) continue;
    const uint32_t bytes = min((uint32_t)c.tokens, 1u << a.block_shift) * a.row_bytes;
    const unsigned char* const from = base + (uint64_t)(uint32_t)c.from * block_bytes;
    unsigned char* const to = base + (uint64_t)(uint32_t)c.to * block_bytes;
    for (uint32_t at = lane * 16u; at < bytes; at += 4096u) {
      // loaded without a branch around them: what lies beyond is the last piece again
      auto piece = [&](uint32_t u) { return *reinterpret_cast<const uint4*>(from + min(at + u * 1024u, bytes - 16u)); };
      auto put = [&](uint32_t u, const uint4& x) { if (at + u * 1024u < bytes) *reinterpret_cast<uint4*>(to + at + u * 1024u) = x; };
      const uint4 x0 = piece(0), x1 = piece(1), x2 = piece(2), x3 = piece(3);
      put(0, x0); put(1, x1); put(2, x2); put(3, x3);
    }
  }
}

uint32_t chunks_of(uint32_t n_blocks) { return (n_blocks + CHUNK - 1) / CHUNK; }
uint64_t up16(uint64_t bytes) { return (bytes + 15) & ~15ull; }

// Where a call's scratch holds what: the counter and the marks, which are zero between calls, then the rest.
uint64_t carve_fork(ForkArgs* a, unsigned char* base, uint32_t n_seq, uint32_t n_blocks, uint32_t max_blocks) {
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t was = at; at += up16(bytes); return base + was; };
  uint32_t* arrived = (uint32_t*)take(16);
  uint32_t* marks = (uint32_t*)take(4ull * n_blocks);
  ForkPlan* plan = (ForkPlan*)take(sizeof(ForkPlan));
  uint32_t* given = (uint32_t*)take(4ull * std::max(n_seq, chunks_of(n_blocks)));
  uint32_t* before = (uint32_t*)take(4ull * n_seq);
  int32_t* copy_of = (int32_t*)take(4ull * n_seq);
  int32_t* taker = (int32_t*)take(4ull * n_seq);
  int32_t* old_lengths = (int32_t*)take(4ull * n_seq);
  int32_t* aside = (int32_t*)take(4ull * std::max<uint64_t>((uint64_t)n_seq * max_blocks, n_blocks));
  if (a) { a->arrived = arrived; a->marks = marks; a->plan = plan; a->given = given; a->before = before; a->copy_of = copy_of; a->taker = taker; a->old_lengths = old_lengths; a->aside = aside; a->place = (uint32_t*)aside; }
  return at;
}

}  // namespace

uint64_t cache_fork_scratch(uint32_t n_seq, uint32_t n_blocks, uint32_t max_blocks) { return carve_fork(nullptr, nullptr, n_seq, n_blocks, max_blocks); }

hipError_t launch_cache_fork(ForkArgs a, void* scratch, hipStream_t st) {
  if (a.n_seq <= SMALL_SEQ && (uint64_t)a.n_seq * a.max_blocks <= SMALL_ENTRIES && a.n_blocks <= SMALL_BLOCKS) {
    const uint32_t lds = (a.n_seq * a.max_blocks + a.n_blocks) * 4;
    if (lds > 48u * 1024) {                       // the limit that all calls have in common
      hipError_t e = hipFuncSetAttribute((const void*)fork_small_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (SMALL_ENTRIES + SMALL_BLOCKS) * 4);
      if (e != hipSuccess) return e;
    }
    fork_small_kernel<<<1, SMALL_THREADS, lds, st>>>(a);
    return hipGetLastError();
  }
  carve_fork(&a, (unsigned char*)scratch, a.n_seq, a.n_blocks, a.max_blocks);
  fork_mark_kernel<<<a.n_seq + 1, THREADS, a.n_seq * 4, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  fork_count_kernel<<<std::min((a.n_seq + WAVES - 1) / WAVES, COUNT_WGS), THREADS, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  fork_write_kernel<<<a.n_seq + a.n_groups, THREADS, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_compact(ForkArgs a, void* scratch, hipStream_t st) {
  carve_fork(&a, (unsigned char*)scratch, a.n_seq, a.n_blocks, a.max_blocks);
  const uint32_t chunks = chunks_of(a.n_blocks);
  compact_mark_kernel<<<a.n_seq, THREADS, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  compact_count_kernel<<<chunks, THREADS, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  compact_place_kernel<<<chunks, THREADS, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  compact_write_kernel<<<a.n_seq + std::min(chunks, 256u), THREADS, 0, st>>>(a);
  return hipGetLastError();
}

constexpr uint32_t COPY_WGS = 4096;
hipError_t launch_cache_copy(const CopyArgs& a, hipStream_t st) {
  if (a.n_copies == 0) return hipSuccess;
  const uint32_t wide = (a.layers * 2 * a.kv_heads + WAVES - 1) / WAVES, high = std::min(a.n_copies, std::max(1u, COPY_WGS / wide));
  copy_blocks_kernel<<<dim3(wide, high), THREADS, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace qzo
