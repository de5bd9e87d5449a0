// Page tables of a serving step, from the lengths of its sequences.
//
// want_s = min(ceil(length_s / page), max_pages); row s gives back entries want_s .. held_s - 1 and lacks entries held_s .. want_s - 1.  Entries are numbered through all rows in
// order.  Entry i of the m given back goes to free_pages[count + m - 1 - i], entry i of those that lack takes free_pages[count + m - 1 - i]: the one undoes the other.
//
// Nothing here is large: a step moves a few pages, and what it takes is a chain of dependent loads.  So one workgroup does all the tables (a thread a sequence, sums over the
// workgroup, then a thread a moved page, found in the sums by bisection in LDS), and writes slots and positions too where tokens are few; many tokens are a
// second launch over the chip, which finds each token's sequence in cu_new.
#include <algorithm>

#include "sb_cache.h"

namespace sb {

constexpr int kPoolThreads = 1024;
struct PoolParams {
  int S, max_pages, num_pages, page_shift;
  int32_t *table, *held, *free_pages, *free_count;
  const int32_t *cached, *added;
  int total_new;
  int32_t *cu, *positions, *missing;
  int64_t* slots;
  int tokens_here;  // slots and positions are this launch's
};

// Sum over the workgroup's threads up to this one (inclusive); `total`: over all.  All threads call it.
template <typename T>
__device__ inline T scan(T x, T* sums, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T t = __shfl_up(x, off, 64);
    if (lane >= off) x += t;
  }
  __syncthreads();  // sums of the scan before have been read
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPoolThreads / 64; ++w) {
    const T t = sums[w];
    if (w < wave) before += t;
    total += t;
  }
  return x + before;
}

// Of n ascending ends, how many are <= x.
template <typename T>
__device__ inline int ends_up_to(const T* ends, int n, int64_t x) {
  int lo = 0;
  while (n > 0) {
    const int half = n >> 1;
    if ((int64_t)ends[lo + half] <= x) { lo += half + 1; n -= half + 1; } else n = half;
  }
  return lo;
}

// Tokens first, first + stride, ..: position and slot.  `cu` [S+1] and the table are complete.
__device__ inline void write_tokens(const PoolParams& P, int64_t first, int64_t stride) {
  for (int64_t t = first; t < P.total_new; t += stride) {
    const int s = ends_up_to(P.cu + 1, P.S, t);
    int64_t pos = 0, slot = -1;
    if (s < P.S) {
      pos = (int64_t)max(P.cached[s], 0) + (t - P.cu[s]);
      const int64_t j = pos >> P.page_shift;
      if (P.slots && j < P.max_pages) {
        const int page = P.table[(int64_t)s * P.max_pages + j];
        if (page >= 0 && page < P.num_pages) slot = ((int64_t)page << P.page_shift) + (pos & ((1 << P.page_shift) - 1));
      }
    }
    if (P.slots) P.slots[t] = slot;
    if (P.positions) P.positions[t] = (int32_t)min(pos, (int64_t)0x7fffffff);
  }
}

__global__ __launch_bounds__(kPoolThreads) void page_tables_kernel(PoolParams P) {
  __shared__ int64_t sums[kPoolThreads / 64];
  __shared__ int64_t ends[kPoolThreads];  // of the moved entries of a chunk's rows
  __shared__ int firsts[kPoolThreads];    // the first of them
  const int tid = threadIdx.x;
  auto row = [&](int s, int& want, int& held) {
    want = held = 0;
    if (s >= P.S) return;
    const int a = P.added[s];
    const int64_t length = a < 0 ? 0 : (int64_t)max(P.cached[s], 0) + a;
    want = (int)min((length + (1 << P.page_shift) - 1) >> P.page_shift, (int64_t)P.max_pages);
    held = min(max(P.held[s], 0), P.max_pages);
  };
  const int64_t count = min(max(P.free_count[0], 0), P.num_pages);
  int64_t back = 0, total;
  for (int s0 = 0; s0 < P.S; s0 += kPoolThreads) {
    int want, held;
    row(s0 + tid, want, held);
    back += max(held - want, 0);
  }
  scan(back, sums, back);  // (all threads: the sum)
  // what goes back
  int64_t before = 0;
  if (back > 0) {
    for (int s0 = 0; s0 < P.S; s0 += kPoolThreads) {
      int want, held;
      row(s0 + tid, want, held);
      const int64_t end = scan((int64_t)max(held - want, 0), sums, total);
      ends[tid] = end;
      firsts[tid] = want;
      __syncthreads();
      for (int64_t i = tid; i < total; i += kPoolThreads) {
        const int r = ends_up_to(ends, kPoolThreads, i);
        const int64_t at = (int64_t)(s0 + r) * P.max_pages + firsts[r] + (i - (r > 0 ? ends[r - 1] : 0));
        const int64_t to = count + back - 1 - (before + i);
        if (to < P.num_pages) P.free_pages[to] = P.table[at];
        P.table[at] = -1;
      }
      before += total;
      __syncthreads();
    }
  }
  const int64_t now = min(count + back, (int64_t)P.num_pages);
  // what lacks, and the new tokens
  __threadfence_block();
  __syncthreads();
  int64_t lacked = 0, tokens = 0;
  if (tid == 0) P.cu[0] = 0;
  for (int s0 = 0; s0 < P.S; s0 += kPoolThreads) {
    const int s = s0 + tid;
    int want, held;
    row(s, want, held);
    const int64_t lack = max(want - held, 0), end = scan(lack, sums, total);
    ends[tid] = end;
    firsts[tid] = held;
    if (s < P.S) {
      const int64_t got = min(max(now - lacked - (end - lack), (int64_t)0), lack);
      if (lack > 0 || want < held) P.held[s] = lack > 0 ? held + (int)got : want;
    }
    __syncthreads();
    for (int64_t i = tid; i < total; i += kPoolThreads) {
      const int r = ends_up_to(ends, kPoolThreads, i);
      const int64_t at = (int64_t)(s0 + r) * P.max_pages + firsts[r] + (i - (r > 0 ? ends[r - 1] : 0));
      const int64_t from = now - 1 - (lacked + i);
      P.table[at] = from >= 0 ? P.free_pages[from] : -1;
    }
    lacked += total;
    const int64_t n = s < P.S ? max(P.added[s], 0) : 0, last = scan(n, sums, total);
    if (s < P.S) P.cu[s + 1] = (int32_t)min(tokens + last, (int64_t)0x7fffffff);
    tokens += total;
  }
  if (tid == 0) {
    P.free_count[0] = (int)max(now - lacked, (int64_t)0);
    if (P.missing) P.missing[0] = (int)min(max(lacked - now, (int64_t)0), (int64_t)0x7fffffff);
  }
  if (P.tokens_here) {
    __threadfence_block();
    __syncthreads();
    write_tokens(P, tid, kPoolThreads);
  }
}

__global__ __launch_bounds__(256) void token_slots_kernel(PoolParams P) { write_tokens(P, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256); }

}  // namespace sb

using namespace sb;

extern "C" int sb_cache_tables(const sb_page_pool* pool, const int32_t* cached, const int32_t* added, int32_t total_new, int32_t* cu_new, int32_t* positions, int64_t* slots,
                               int32_t* missing, void* stream) {
  if (!pool) { set_error("null pool"); return SB_ERR_INVALID_ARG; }
  if (pool->num_seqs < 0 || pool->max_pages < 0 || pool->num_pages < 0 || total_new < 0) { set_error("negative size"); return SB_ERR_INVALID_ARG; }
  if (pool->page_size < 16 || pool->page_size > 1024 || (pool->page_size & (pool->page_size - 1)) != 0) {
    set_error("page_size %d unsupported (a power of two, 16 .. 1024)", pool->page_size);
    return SB_ERR_UNSUPPORTED;
  }
  if ((int64_t)pool->max_pages * pool->page_size > 0x7fffffffll - 1024) { set_error("max_pages * page_size passes 32 bits"); return SB_ERR_UNSUPPORTED; }
  if (!cu_new || !pool->free_count || (pool->num_pages > 0 && !pool->free_pages)) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if (pool->num_seqs > 0 && (!cached || !added || !pool->held || (pool->max_pages > 0 && !pool->page_table))) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  PoolParams P{};
  P.S = pool->num_seqs; P.max_pages = pool->max_pages; P.num_pages = pool->num_pages; P.page_shift = __builtin_ctz((unsigned)pool->page_size);
  P.table = pool->page_table; P.held = pool->held; P.free_pages = pool->free_pages; P.free_count = pool->free_count;
  P.cached = cached; P.added = added; P.cu = cu_new; P.positions = positions; P.slots = slots; P.missing = missing;
  P.total_new = positions || slots ? total_new : 0;
  P.tokens_here = P.total_new <= 4 * kPoolThreads;
  const hipStream_t st = (hipStream_t)stream;
  KernelTimer kt(K_PLAN, st);
  hipLaunchKernelGGL(page_tables_kernel, dim3(1), dim3(kPoolThreads), 0, st, P);
  SB_LAUNCH_CHECK("page_tables_kernel");
  if (!P.tokens_here) {
    hipLaunchKernelGGL(token_slots_kernel, dim3((unsigned)std::min<int64_t>(((int64_t)P.total_new + 255) / 256, 4096)), dim3(256), 0, st, P);
    SB_LAUNCH_CHECK("token_slots_kernel");
  }
  return SB_OK;
}
