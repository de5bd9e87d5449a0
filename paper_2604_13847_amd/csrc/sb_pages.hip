// Page tables of a serving step, from the lengths of its sequences.
//
// want_s = min(ceil(length_s / page), max_pages); row s gives back entries want_s .. held_s - 1 and lacks entries held_s .. want_s - 1.  Entries are numbered through all rows in
// order.  Entry i of the m given back goes to free_pages[count + m - 1 - i], entry i of those that lack takes free_pages[count + m - 1 - i]: the one undoes the other.
//
// Nothing here is large: a step moves a few pages, and what it takes is a chain of dependent loads.  So one workgroup does all the tables (a thread a sequence, sums over the
// workgroup, then a thread a moved page, found in the sums by bisection in LDS, four at a time), and writes slots and positions too where tokens are few; many tokens are a
// second launch over the chip, which finds each token's sequence in cu_new.  Of few sequences the workgroup is small: its barriers are cheaper.
// 64 sequences with four tokens each, one in 16 finished: 3.8 us on the GPU (host and launch 9).  1000 with 8 prompts of 12288 to 16384 tokens, pages of 16: 10 us and 4.6 for the tokens' slots; by scans through
// LDS and one entry a thread at a time it was 17.
#include <algorithm>
#include <type_traits>

#include "sb_cache.h"

namespace sb {

struct PoolParams {
  int S, max_pages, num_pages, page_shift;
  int32_t *table, *held, *free_pages, *free_count;
  const int32_t *cached, *added;
  int total_new;
  int32_t *cu, *positions, *missing;
  int64_t* slots;
  int tokens_here;  // slots and positions are this launch's
};

// Of n ascending ends, how many are <= x.
__device__ inline int ends_up_to(const int32_t* ends, int n, int64_t x) {
  int lo = 0;
  while (n > 0) {
    const int half = n >> 1;
    if ((int64_t)ends[lo + half] <= x) { lo += half + 1; n -= half + 1; } else n = half;
  }
  return lo;
}
// The same of N ends (a power of two), fewer than N of them <= x: without branches, so that several run side by side.
template <int N>
__device__ inline int ends_up_to(const int32_t* ends, int32_t x) {
  int lo = 0;
#pragma unroll
  for (int step = N / 2; step > 0; step >>= 1) lo += ends[lo + step - 1] <= x ? step : 0;
  return lo;
}
constexpr int64_t kMost = 0x7fffffff;  // entries that move: no more than there are pages

// Tokens first, first + stride, ..: position and slot.  The table is complete; ends [S]: cu_new without its zero.
__device__ inline void write_tokens(const PoolParams& P, const int32_t* ends, const int32_t* cached, int64_t first, int64_t stride) {
  for (int64_t t = first; t < P.total_new; t += stride) {
    const int s = ends_up_to(ends, P.S, t);
    int64_t pos = 0, slot = -1;
    if (s < P.S) {
      pos = (int64_t)max(cached[s], 0) + (t - (s > 0 ? ends[s - 1] : 0));
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

// Sums of three numbers over the workgroup's threads up to this one (inclusive), and over all.  Sums that pass 32 bits stop at 2^32 - 1.  All threads call it.
struct Three { unsigned x[3]; };
__device__ inline unsigned add_up(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }
// x of the lane CTRL says, 0 where there is none or the lane's row of 16 is not in ROWS
template <int CTRL, int ROWS> __device__ inline unsigned moved(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false); }
__device__ inline unsigned scan_row(unsigned x) {  // of 16 lanes
  x = add_up(x, moved<0x111, 0xf>(x));
  x = add_up(x, moved<0x112, 0xf>(x));
  x = add_up(x, moved<0x114, 0xf>(x));
  return add_up(x, moved<0x118, 0xf>(x));
}
template <int THREADS>
__device__ inline Three scan(Three v, unsigned (&sums)[3][16], Three& total) {
  static_assert(THREADS <= 1024, "a row of lanes holds the wavefronts' sums");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    v.x[i] = scan_row(v.x[i]);
    v.x[i] = add_up(v.x[i], moved<0x142, 0xa>(v.x[i]));  // the row before, for every second row
    v.x[i] = add_up(v.x[i], moved<0x143, 0xc>(v.x[i]));  // the first half, for the second
  }
  __syncthreads();  // sums of the scan before have been read
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < 3; ++i) sums[i][wave] = v.x[i];
  __syncthreads();
  const unsigned waves = scan_row(lane < 48 && (lane & 15) < THREADS / 64 ? sums[lane >> 4][lane & 15] : 0);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    total.x[i] = (unsigned)__builtin_amdgcn_readlane((int)waves, 16 * i + 15);
    if (wave > 0) v.x[i] = add_up(v.x[i], (unsigned)__builtin_amdgcn_readlane((int)waves, 16 * i + wave - 1));
  }
  return v;
}

// body(n, i) for this thread's part of 0 .. moved - 1: entries i, i + THREADS, .. of n, which may pass the last one
template <int THREADS, typename F>
__device__ inline void batches(int64_t moved, F body) {
  int64_t i = threadIdx.x;
  for (; i - threadIdx.x + THREADS < moved; i += 4 * THREADS) body(std::integral_constant<int, 4>(), i);
  if (i < moved) body(std::integral_constant<int, 1>(), i);
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void page_tables_kernel(PoolParams P) {
  __shared__ unsigned sums[3][16];
  __shared__ int32_t ends[THREADS];  // of the moved entries of a chunk's rows
  __shared__ int firsts[THREADS];    // the first of them
  __shared__ int32_t cu[THREADS], have[THREADS];
  const int tid = threadIdx.x;
  struct Row { int want, held, said, added, cached; };  // said: held as it stands in memory
  auto row = [&](int s) {
    Row r{};
    if (s >= P.S) return r;
    r.added = P.added[s];
    r.cached = max(P.cached[s], 0);
    r.said = P.held[s];
    const int64_t length = r.added < 0 ? 0 : (int64_t)r.cached + r.added;
    r.want = (int)min((length + (1 << P.page_shift) - 1) >> P.page_shift, (int64_t)P.max_pages);
    r.held = min(max(r.said, 0), P.max_pages);
    return r;
  };
  auto sums_of = [&](const Row& r) { return Three{{(unsigned)max(r.held - r.want, 0), (unsigned)max(r.want - r.held, 0), (unsigned)max(r.added, 0)}}; };  // given back, lacking, new tokens
  // entry i of a chunk's moved ones
  auto entry = [&](int s0, int32_t i) {
    const int r = ends_up_to<THREADS>(ends, i);
    return (int64_t)(s0 + r) * P.max_pages + firsts[r] + (i - (r > 0 ? ends[r - 1] : 0));
  };
  const int64_t count = min(max(P.free_count[0], 0), P.num_pages);
  const bool one = P.S <= THREADS;  // all sequences at once: their numbers stay in registers
  Row mine = row(tid);
  Three all{}, chunk = scan<THREADS>(sums_of(mine), sums, all);
  const Three first_chunk = all;
  if (!one) {
    Three more{};
    for (int s = tid + THREADS; s < P.S; s += THREADS) {
      const Three t = sums_of(row(s));
#pragma unroll
      for (int i = 0; i < 3; ++i) more.x[i] = add_up(more.x[i], t.x[i]);
    }
    scan<THREADS>(more, sums, more);
#pragma unroll
    for (int i = 0; i < 3; ++i) all.x[i] = add_up(all.x[i], more.x[i]);
  }
  const int64_t back = min((int64_t)all.x[0], kMost);
  if (back > 0) {  // what goes back
    int64_t before = 0;
    for (int s0 = 0; s0 < P.S; s0 += THREADS) {
      Row r = mine;
      Three c = chunk, total = first_chunk;
      if (s0 > 0) {
        r = row(s0 + tid);
        c = scan<THREADS>(sums_of(r), sums, total);
      }
      ends[tid] = (int32_t)min((int64_t)c.x[0], kMost);
      firsts[tid] = r.want;
      __syncthreads();
      const int64_t moved = min((int64_t)total.x[0], back - before);
      batches<THREADS>(moved, [&](auto n, int64_t i0) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
        int64_t at[N];
        int page[N];
#pragma unroll
        for (int b = 0; b < N; ++b) {
          at[b] = entry(s0, (int32_t)min(i0 + b * THREADS, moved - 1));
          page[b] = P.table[at[b]];
        }
#pragma unroll
        for (int b = 0; b < N; ++b) {
          const int64_t i = i0 + b * THREADS, to = count + back - 1 - (before + i);
          if (i >= moved) continue;
          if (to < P.num_pages) P.free_pages[to] = page[b];
          P.table[at[b]] = -1;
        }
      });
      before += total.x[0];
      __syncthreads();
    }
    __threadfence_block();  // (what went back is read below by other threads)
    __syncthreads();
  }
  const int64_t now = min(count + back, (int64_t)P.num_pages);
  int64_t lacked = 0, tokens = 0;  // of the chunks before
  if (tid == 0) P.cu[0] = 0;
  for (int s0 = 0; s0 < P.S; s0 += THREADS) {  // what lacks, and the new tokens
    const int s = s0 + tid;
    Row r = mine;
    Three c = chunk, total = first_chunk;
    if (s0 > 0) {
      r = row(s);
      c = scan<THREADS>(sums_of(r), sums, total);  // (its barriers: the entries of the chunk before are done)
    }
    const int64_t lack = max(r.want - r.held, 0);
    ends[tid] = (int32_t)min((int64_t)c.x[1], kMost);
    firsts[tid] = r.held;
    const int32_t end = (int32_t)min(tokens + c.x[2], (int64_t)0x7fffffff);
    if (s < P.S) {
      const int64_t got = min(max(now - lacked - ((int64_t)c.x[1] - lack), (int64_t)0), lack);
      if (r.want != r.said) P.held[s] = lack > 0 ? r.held + (int)got : r.want;
      P.cu[s + 1] = end;
    }
    if (one) {
      cu[tid] = end;
      have[tid] = r.cached;
    }
    __syncthreads();
    const int64_t moved = min((int64_t)total.x[1], max(now - lacked, (int64_t)0));  // (what lacks for want of pages is -1 already)
    batches<THREADS>(moved, [&](auto n, int64_t i0) __attribute__((always_inline)) {
      constexpr int N = decltype(n)::value;
      int64_t at[N];
      int page[N];
#pragma unroll
      for (int b = 0; b < N; ++b) {
        const int64_t i = min(i0 + b * THREADS, moved - 1);
        page[b] = P.free_pages[now - 1 - (lacked + i)];
        at[b] = entry(s0, (int32_t)i);
      }
#pragma unroll
      for (int b = 0; b < N; ++b)
        if (i0 + b * THREADS < moved) P.table[at[b]] = page[b];
    });
    lacked += total.x[1];
    tokens += total.x[2];
  }
  if (tid == 0) {
    P.free_count[0] = (int)max(now - lacked, (int64_t)0);
    if (P.missing) P.missing[0] = (int)min(max(lacked - now, (int64_t)0), (int64_t)0x7fffffff);
  }
  if (P.tokens_here) {
    __threadfence_block();
    __syncthreads();
    if (one) write_tokens(P, cu, have, tid, THREADS);
    else write_tokens(P, P.cu + 1, P.cached, tid, THREADS);
  }
}

__global__ __launch_bounds__(256) void token_slots_kernel(PoolParams P) {
  write_tokens(P, P.cu + 1, P.cached, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

}  // namespace sb

using namespace sb;

extern "C" int sb_cache_tables(const sb_page_pool* pool, const int32_t* cached, const int32_t* added, int32_t total_new, int32_t* cu_new, int32_t* positions, int64_t* slots,
                               int32_t* missing, void* stream) {
  if (!pool) { set_error("null pool"); return SB_ERR_INVALID_ARG; }
  if (pool->num_seqs < 0 || pool->max_pages < 0 || pool->num_pages < 0 || ((positions || slots) && total_new < 0)) { set_error("negative size"); return SB_ERR_INVALID_ARG; }
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
  P.tokens_here = P.total_new <= 4096;  // (four a thread; a launch of their own costs 4 us)
  const hipStream_t st = (hipStream_t)stream;
  KernelTimer kt(K_PLAN, st);
  if (P.S <= 256 && P.total_new <= 1024) hipLaunchKernelGGL(page_tables_kernel<256>, dim3(1), dim3(256), 0, st, P);
  else hipLaunchKernelGGL(page_tables_kernel<1024>, dim3(1), dim3(1024), 0, st, P);
  SB_LAUNCH_CHECK("page_tables_kernel");
  if (!P.tokens_here) {
    hipLaunchKernelGGL(token_slots_kernel, dim3((unsigned)std::min<int64_t>(((int64_t)P.total_new + 255) / 256, 4096)), dim3(256), 0, st, P);
    SB_LAUNCH_CHECK("token_slots_kernel");
  }
  return SB_OK;
}
