// Attention of new tokens over a paged cache (serving).
//
// Whole chunks of a prompt go through the kernel of packed batches (sb_window.hip), which looks its key tiles up in the page table.  Few rows a sequence (single tokens above
// all) are another matter: every key is read for a handful of products, so what bounds them is memory, and what fills the chip is splitting the keys.  cache_split_kernel
// gives each (sequence, KV head, run of keys) to a workgroup of two wavefronts that stage their own strips and never wait for each other until they add up at the
// end; cache_merge_kernel joins the runs.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sb_window.h"

namespace sb {

int check_cache(const sb_cache* c, const sb_chunk* n) {
  if (!c || !n) { set_error("null cache or chunk"); return SB_ERR_INVALID_ARG; }
  if (c->dtype != SB_BF16 && c->dtype != SB_F32) { set_error("dtype must be SB_BF16 or SB_F32"); return SB_ERR_INVALID_ARG; }
  if (c->num_pages < 0 || c->max_pages < 0 || n->num_seqs < 0 || n->total_new < 0 || n->max_new < 0 || n->max_length < 0) {
    set_error("negative size");
    return SB_ERR_INVALID_ARG;
  }
  if (c->num_kv_heads < 1 || n->num_q_heads < 1 || n->num_q_heads % c->num_kv_heads != 0) {
    set_error("num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)", n->num_q_heads, c->num_kv_heads);
    return SB_ERR_INVALID_ARG;
  }
  if (c->head_dim != 64 && c->head_dim != 128) { set_error("head_dim %d unsupported (64 or 128)", c->head_dim); return SB_ERR_UNSUPPORTED; }
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0) {
    set_error("page_size %d unsupported (a power of two, 16 .. 1024)", c->page_size);
    return SB_ERR_UNSUPPORTED;
  }
  if ((int64_t)c->max_pages * c->page_size > 0x7fffffffll - 1024) { set_error("max_pages * page_size passes 32 bits"); return SB_ERR_UNSUPPORTED; }
  return SB_OK;
}
int check_cache_arrays(const sb_cache* c, const sb_chunk* n) {
  if (!n->cu_new || !n->cached) { set_error("cu_new and cached are required"); return SB_ERR_INVALID_ARG; }
  if ((c->num_pages > 0 && (!c->k || !c->v)) || (c->max_pages > 0 && !c->page_table)) { set_error("pages without an address"); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}
PagedCache make_paged(const sb_cache* c) {
  return PagedCache{c->k, c->v, c->page_table, c->num_pages, c->max_pages, c->page_size, __builtin_ctz((unsigned)c->page_size), c->num_kv_heads};
}

static int check_cache_attn(const sb_cache* c, const sb_chunk* n, int32_t window, int32_t sinks) {
  const int rc = check_cache(c, n);
  if (rc != SB_OK) return rc;
  if (window < 1 || sinks < 0) { set_error("window (%d) must be at least 1 and sinks (%d) not negative", window, sinks); return SB_ERR_INVALID_ARG; }
  return check_rows(n->total_new, n->num_q_heads / c->num_kv_heads);
}

// ---------------------------------------------------------------------------------------------
// Few rows (bfloat16): an item is up to 32 flattened rows of a KV head and per_split strips of 32 keys; a wavefront takes every second strip.  A wavefront's
// strips of K and V come by buffer loads straight into its own LDS, the next strip's while one is worked on: 64 KiB a CU on their way (head_dim 128), no barrier, and the
// products of a strip take a quarter of the time that memory takes to deliver four.  Pages are looked up 64 strips ahead, a lane a strip.
// 64 sequences of 500 to 32768 tokens, 32/8 heads: 0.39 ms, 5.1 TB/s, where a copy of 2 GiB reaches 4.95 (workgroups of four wavefronts, one a CU: 0.50 ms).  One sequence of 4097 tokens: 8.6 us (four wavefronts: 12)
// and 4 to join, a chain of dependent loads (lengths, page, keys) behind the launch.
// Two wavefronts: two such workgroups share a CU's LDS, and one's start and end are hidden by the other's stream.
template <int D>
__global__ __launch_bounds__(128) void cache_split_kernel(WindowParams P) {
  constexpr int NW = 2;
  constexpr int ROW_B = D * 2, STRIP_B = 32 * ROW_B, NOP = D / 16, C = D / 8, RPI = 64 / C, LPG = 16 / RPI;  // loads per 16 rows
  constexpr int OUT_P = D + 4;  // floats from row to row of a wavefront's sums in LDS
  __shared__ __attribute__((aligned(1024))) char ring[NW][2][2 * STRIP_B];  // K, V
  __shared__ float stats[2][NW][32];
  static_assert(32 * OUT_P * 4 <= 4 * STRIP_B, "the sums take the strips' place");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  // (what follows a division is the same in every lane but lies in vector registers, where what the loads' resources are made of must not come from)
  const int z = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (unsigned)P.Hkv % (unsigned)P.splits));
  const RowTile t = locate_tile<kSplitRows, true>(P, blockIdx.x / (unsigned)P.Hkv / (unsigned)P.splits);
  if (t.s < 0) return;
  const int g = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % (unsigned)P.Hkv));
  const int rows = t.n * P.G, m0 = t.tile * kSplitRows, mine = min(rows - m0, kSplitRows);
  auto token = [&](int m) { return (int)((unsigned)min(m, rows - 1) / (unsigned)P.G); };
  const int i = token(m0 + l32), h = g * P.G + min(m0 + l32, rows - 1) - i * P.G, pos = t.pos0 + i;
  const int ta = __builtin_amdgcn_readfirstlane(t.pos0 + token(m0)), last = __builtin_amdgcn_readfirstlane(t.pos0 + token(m0 + 31));
  const int tb = min(last, P.cache.max_pages * P.cache.page_size - 1), end = tb + 1, lo = max(0, ta - P.window + 1);
  const KeyTiles<32> strips(ta, tb, P.window, P.sinks);
  const int begin = (int)min((int64_t)z * P.per_split, (int64_t)strips.count());
  const int count = z < P.splits - 1 ? min(begin + P.per_split, strips.count()) : strips.count();
  const int turns = (count - begin - wave + NW - 1) / NW;  // strips of this wavefront: begin + wave + NW x (may be none)
  const int32_t* const table = P.cache.table + (int64_t)t.s * P.cache.max_pages;
  const unsigned page_b = (unsigned)P.Hkv << P.cache.page_shift;  // rows of a page

  // Of strip begin + wave + NW (x0 + lane): the first row, in units of 16 rows, of its keys 0 .. 15 and 16 .. 31 in the cache, and how many of each exist; -1, 0: none
  int where[2], there[2], x0 = 0;
  auto look_up = [&](int from) __attribute__((always_inline)) {
    x0 = from;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      where[b] = 0;
      there[b] = 0;
      if (from + lane < turns) {
        const int u = 32 * strips.at(begin + wave + NW * (from + lane)) + 16 * b;
        if (u < end && (u + 16 > lo || u < P.sinks)) {
          const int page = table[u >> P.cache.page_shift];
          if ((unsigned)page < (unsigned)P.cache.num_pages) {
            there[b] = min(end - u, 16);
            where[b] = page;
          }
        }
      }
    }
  };
  unsigned voff[LPG];
#pragma unroll
  for (int a = 0; a < LPG; ++a) {
    const int r = a * RPI + lane / C;  // (the swizzle repeats every 16 rows)
    voff[a] = (unsigned)(r * ROW_B + 16 * ((lane % C) ^ chunk_swizzle<D>(r)));
  }
  const unsigned ring0 = lds_offset(&ring[wave][0][0]);
  const unsigned long long head = ((unsigned long long)g << P.cache.page_shift) * ROW_B;
  auto issue = [&](int x) __attribute__((always_inline)) {  // strip x of this wavefront, or, past its last, as many loads of nothing
    const unsigned slot = ring0 + (x & 1) * 2 * STRIP_B;
    const int at = min(x - x0, 63);
    const int u = __builtin_amdgcn_readfirstlane(32 * strips.at(min(begin + wave + NW * x, max(strips.count() - 1, 0))));
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const unsigned page = (unsigned)__builtin_amdgcn_readlane(where[b], at);
      const int n = x < turns ? __builtin_amdgcn_readlane(there[b], at) : 0;
      const unsigned long long o = head + ((unsigned long long)page * page_b + ((u + 16 * b) & (P.cache.page_size - 1))) * ROW_B;
      const unsigned bytes = (unsigned)n * ROW_B;
      const i32x4 rk = QuadLoader<D>::resource((unsigned long long)P.cache.k + o, bytes), rv = QuadLoader<D>::resource((unsigned long long)P.cache.v + o, bytes);
#pragma unroll
      for (int a = 0; a < LPG; ++a)
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" : : "v"(voff[a]), "s"(slot + b * 16 * ROW_B + a * 1024), "s"(rk) : "memory", "m0");
#pragma unroll
      for (int a = 0; a < LPG; ++a)
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" : : "v"(voff[a]), "s"(slot + STRIP_B + b * 16 * ROW_B + a * 1024), "s"(rv) : "memory", "m0");
    }
  };

  // B operand of S^T = K Q^T: column = row lane%32, slots = d 16ks + 8hf + (0..7)
  bf16x8 qf[NOP];
  {
    const bf16* qp = (const bf16*)P.q + ((int64_t)(t.row0 + i) * P.Hq + h) * D + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  float top = -__builtin_inff(), l = 0.f;  // largest score, in units of log 2, and sum
  if (turns > 0) {
    look_up(0);
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) asm volatile("" : "+v"(qf[ks]));
    asm volatile("" : "+v"(where[0]), "+v"(where[1]), "+v"(there[0]), "+v"(there[1]));
    issue(0);
  }
  unsigned row_a[NOP], tr_a[D / 32][2];
#pragma unroll
  for (int ks = 0; ks < NOP; ++ks) row_a[ks] = ring0 + l32 * ROW_B + 16 * ((2 * ks + hf) ^ chunk_swizzle<D>(l32));
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = 8 * half + 4 * hf + ((lane & 15) >> 2), d = 32 * dt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      tr_a[dt][half] = ring0 + STRIP_B + r * ROW_B + 16 * ((d >> 3) ^ chunk_swizzle<D>(r)) + 2 * (d & 7);
    }
  for (int x = 0; x < turns; ++x) {
    const int u0 = 32 * strips.at(begin + wave + NW * x);
    const unsigned off = (x & 1) * 2 * STRIP_B;
    const unsigned have = (1u << __builtin_amdgcn_readlane(there[0], x - x0)) - 1 | ((1u << __builtin_amdgcn_readlane(there[1], x - x0)) - 1) << 16;  // keys that exist
    const bool refill = x + 1 < turns && x + 1 - x0 == 64;
    if (refill) look_up(x + 1);
    if (refill) asm volatile("s_waitcnt vmcnt(0)" : "+v"(where[0]), "+v"(where[1]), "+v"(there[0]), "+v"(there[1]) : : "memory");
    issue(x + 1);
    wait_vmcnt<4 * LPG>();  // strip x has landed
    bf16x8 op[NOP];
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) op[ks] = *(const bf16x8 __attribute__((address_space(3)))*)(uintptr_t)(row_a[ks] + off);
    f32x16 sc = zero16();
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) sc = mfma32(op[ks], qf[ks], sc);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        const unsigned o = off + kk * 16 * ROW_B;
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(tr_a[dt][0] + o));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(tr_a[dt][1] + o));
        op[kk * (D / 32) + dt] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    float p[16], mx = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] = sc[v] * P.scale_log2e;
    if (u0 + 31 > ta || (last - u0 >= P.window && u0 + 31 >= P.sinks) || have != ~0u) {
      const Sight sees(pos, u0, hf, P.window, P.sinks);
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (!sees(c_row(v, 0)) || !(have >> c_row(v, hf) & 1)) p[v] = -__builtin_inff();
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, p[v]);
    mx = fmaxf(top, max_across_halves(mx));
    const float ref = mx == -__builtin_inff() ? 0.f : mx;  // nothing seen yet: keep the exponents finite
    const float alpha = fast_exp2(top - ref);
    top = mx;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[dt][v] *= alpha;
    bf16x8 w[2];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float e = fast_exp2(p[v] - ref);
      l += e;  // (before the rounding: LSE keeps float32's precision)
      w[v >> 3][v & 7] = (bf16)e;
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) acc[dt] = mfma32(op[kk * (D / 32) + dt], w[kk], acc[dt]);
  }
  wait_vmcnt<0>();
  // the wavefronts' sums, through LDS (each in its own strips' place)
  l += __shfl_xor(l, 32, 64);
  float* const out = (float*)&ring[wave][0][0];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int vg = 0; vg < 4; ++vg)
      *(f32x4*)(out + l32 * OUT_P + 32 * dt + 8 * vg + 4 * hf) = f32x4{acc[dt][4 * vg], acc[dt][4 * vg + 1], acc[dt][4 * vg + 2], acc[dt][4 * vg + 3]};
  if (hf == 0) { stats[0][wave][l32] = top; stats[1][wave][l32] = l; }
  __syncthreads();
  constexpr int LANES = D / 4;
  const int c = threadIdx.x % LANES;
  for (int r = threadIdx.x / LANES; r < mine; r += 64 * NW / LANES) {
    float best = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) best = fmaxf(best, stats[0][w][r]);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (stats[1][w][r] == 0.f) continue;
      const float f = fast_exp2(stats[0][w][r] - best);
      sum += f * stats[1][w][r];
      x += f * *(const f32x4*)((const float*)&ring[w][0][0] + r * OUT_P + 4 * c);
    }
    const int j = token(m0 + r), hh = g * P.G + m0 + r - j * P.G;
    const int64_t row = (int64_t)(t.row0 + j) * P.Hq + hh;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum, lse2 = sum == 0.f ? -__builtin_inff() : best + __builtin_log2f(sum);  // (a sum that is no number is passed on)
    x *= inv;
    if (P.splits > 1) {
      const int64_t at = ((int64_t)z * P.part_rows + (P.part_seq_rows > 0 ? t.s * P.part_seq_rows : t.row0) + j) * P.Hq + hh;
      if (c == 0) P.part_lse[at] = lse2;
      if (sum != 0.f) *(f32x4*)(P.part_o + at * D + 4 * c) = x;
    } else {
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (bf16)x[e];
      *(bf16x4*)((bf16*)P.o + row * D + 4 * c) = y;
      if (c == 0) P.lse[(int64_t)hh * P.T + t.row0 + j] = lse2 * 0.69314718055994531f;
    }
  }
}

// Joins the runs of keys of the sequences that a launch before had: a workgroup to a row and head, every fourth run a wavefront's.  A run that saw nothing has left LSE -infinity and no
// sums; one that saw what is no number has left that, and so is the row's result.  seq_rows > 0: workgroups for that many rows of every sequence, else for all rows.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_merge_kernel(WindowParams P, int seq_rows) {
  constexpr int E = D / 64;
  __shared__ float sums[4][E + 2][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = (int)(blockIdx.x % (unsigned)P.Hq), at = (int)(blockIdx.x / (unsigned)P.Hq);
  const int s = seq_rows > 0 ? at / seq_rows : sequence_of(P.cu, P.S, at, lane);
  if (s >= P.S) return;  // a row of no sequence: left as it was
  const int row0 = min(max(P.cu[s], 0), P.T), n = min(min(P.cu[s + 1], P.T) - row0, P.max_new), tok = seq_rows > 0 ? row0 + at % seq_rows : at;
  if (tok - row0 < 0 || tok - row0 >= n || n * P.G < P.rows_from || n * P.G > P.rows_to) return;
  const int splits = P.splits;
  const int64_t all = (int64_t)P.part_rows * P.Hq, row = (int64_t)(P.part_seq_rows > 0 ? s * P.part_seq_rows + tok - row0 : tok) * P.Hq + h;
  constexpr int kRuns = 8;  // on their way at a time
  float x[E] = {}, best = -__builtin_inff(), sum = 0.f;
  for (int z0 = wave; z0 < splits; z0 += 4 * kRuns) {
    float lse[kRuns], part[kRuns][E], top = best;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {  // (past the last run, it again)
      const int z = min(z0 + 4 * i, splits - 1);
      lse[i] = P.part_lse[z * all + row];
#pragma unroll
      for (int e = 0; e < E; ++e) part[i][e] = P.part_o[(z * all + row) * D + E * lane + e];
      if (z0 + 4 * i >= splits) lse[i] = -__builtin_inff();
    }
#pragma unroll
    for (int i = 0; i < kRuns; ++i) top = fmaxf(top, lse[i]);
    const float ref = top == -__builtin_inff() ? 0.f : top;  // nothing seen yet: keep the exponents finite
    const float old = fast_exp2(best - ref);
    sum *= old;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= old;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const float f = fast_exp2(lse[i] - ref);
      sum += f;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(f, lse[i] == -__builtin_inff() ? 0.f : part[i][e], x[e]);  // (a run without sums holds whatever was there)
    }
    best = top;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) sums[wave][e][lane] = x[e];
  sums[wave][E][lane] = best;
  sums[wave][E + 1][lane] = sum;
  __syncthreads();
  if (wave > 0) return;
  best = -__builtin_inff();
#pragma unroll
  for (int w = 0; w < 4; ++w) best = fmaxf(best, sums[w][E][lane]);
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.f;
  const float ref = best == -__builtin_inff() ? 0.f : best;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = fast_exp2(sums[w][E][lane] - ref);
    sum += f * sums[w][E + 1][lane];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(f, sums[w][e][lane], x[e]);
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
  for (int e = 0; e < E; ++e) ((T*)P.o)[((int64_t)tok * P.Hq + h) * D + E * lane + e] = (T)(x[e] * inv);
  if (lane == 0) P.lse[(int64_t)h * P.T + tok] = sum == 0.f ? -__builtin_inff() : (best + __builtin_log2f(sum)) * 0.69314718055994531f;
}

int launch_cache_merge(const WindowParams& P, int D, int dtype, dim3 workgroups, int seq_rows, hipStream_t st) {
  auto launch = [&](auto t, auto d) { hipLaunchKernelGGL((cache_merge_kernel<decltype(t), decltype(d)::value>), workgroups, dim3(256), 0, st, P, seq_rows); };
  auto with_d = [&](auto t) { if (D == 128) launch(t, std::integral_constant<int, 128>()); else launch(t, std::integral_constant<int, 64>()); };
  if (dtype == SB_F32) with_d(float()); else with_d(bf16());
  SB_LAUNCH_CHECK("cache_merge_kernel");
  return SB_OK;
}

// How the work is cut.  Sequences of up to kFewRows flattened rows are cache_split_kernel's (bfloat16), the others the packed batches' kernel's; a batch of one kind costs one launch.
constexpr int kFewRows = 2 * kSplitRows;
static int few_seq_rows(int G, int max_new) { return std::min(kFewRows / G, max_new); }  // tokens of such a sequence, at most
struct CacheLaunch {
  int64_t items;          // tiles of rows
  int splits, per_split;  // keys in `splits` runs of per_split tiles
  int part_rows, part_seq_rows;
};
struct CachePlan {
  CacheLaunch few, many;           // items 0: no such launch
  size_t part_o, part_lse, bytes;  // workspace
};
static CachePlan plan_cache(const sb_cache* c, const sb_chunk* n, int window, int sinks) {
  CachePlan p{};
  const int G = n->num_q_heads / c->num_kv_heads, S = n->num_seqs;
  const int64_t most = (int64_t)(n->max_new < n->total_new ? n->max_new : n->total_new) * G;  // rows of a sequence
  auto launch = [&](int64_t most_rows, int rows, int tile, int64_t wanted, int64_t least, int64_t largest) {
    CacheLaunch l{};
    const int64_t by_total = row_tiles_most(n->total_new, S, G, rows), by_seq = (most_rows + rows - 1) / rows * S;
    l.items = by_total < by_seq ? by_total : by_seq;
    // key tiles of an item, about: what max_length, the page table, the window and the sinks leave
    const int64_t in_window = (int64_t)window + (rows + G - 1) / G + sinks + 2 * tile;
    const int64_t longest = std::min<int64_t>(n->max_length, (int64_t)c->max_pages * c->page_size);
    const int64_t keys = std::min(in_window, longest), tiles = (keys + tile - 1) / tile;
    int64_t per = (tiles * l.items * c->num_kv_heads + wanted - 1) / wanted;
    per = (per + least - 1) / least * least;
    if (per < least) per = least;
    if (per > largest) per = largest;
    l.splits = (int)((tiles + per - 1) / per);
    if (l.splits < 1) l.splits = 1;
    l.per_split = (int)per;
    return l;
  };
  p.few.splits = p.many.splits = 1;
  const bool f32 = c->dtype == SB_F32;
  // Two workgroups a CU; a strip for each wavefront at least, and 1024 keys at most, so that sequences of unequal lengths even out.
  if (!f32 && G <= kFewRows && (S > 1 || most <= kFewRows)) p.few = launch(most < kFewRows ? most : kFewRows, kSplitRows, 32, 512, 2, 32);
  // A workgroup a CU (float32, where one takes 32 rows: four), of 8 tiles at least.
  if (f32 || most > kFewRows) p.many = launch(most, forward_rows(c->dtype), f32 ? 32 : 64, f32 ? 1024 : 256, 8, 1 << 30);
  p.few.part_rows = p.many.part_rows = n->total_new;
  // Sums of few rows are laid out by sequence where that is less: a prompt in the batch has none (64 sequences of 32768 tokens, one of them with 8192 new ones: 0.54 GB and not 4.4)
  const int seq_rows = few_seq_rows(G, n->max_new);
  if ((int64_t)seq_rows * S < n->total_new) {
    p.few.part_seq_rows = seq_rows;
    p.few.part_rows = seq_rows * S;
  }
  size_t most_sums = 0;
  for (const CacheLaunch* l : {&p.few, &p.many})
    if (l->splits > 1) most_sums = std::max(most_sums, (size_t)l->splits * l->part_rows * n->num_q_heads);
  p.part_o = align_up(most_sums * sizeof(float));
  p.bytes = align_up(p.part_o + most_sums * c->head_dim * sizeof(float));
  return p;
}

}  // namespace sb

using namespace sb;

extern "C" {

int sb_cache_attn_ws_bytes(const sb_cache* c, const sb_chunk* n, int32_t window, int32_t sinks, int64_t* bytes) {
  if (!bytes) { set_error("null output"); return SB_ERR_INVALID_ARG; }
  const int rc = check_cache_attn(c, n, window, sinks);
  if (rc != SB_OK) return rc;
  *bytes = n->num_seqs == 0 || n->max_new == 0 ? 0 : (int64_t)plan_cache(c, n, window, sinks).bytes;
  return SB_OK;
}

int sb_cache_attn(const sb_cache* c, const sb_chunk* n, int32_t window, int32_t sinks, const void* q, void* o, float* lse, void* ws, void* stream) {
  int rc = check_cache_attn(c, n, window, sinks);
  if (rc != SB_OK) return rc;
  if (n->total_new == 0 || n->num_seqs == 0 || n->max_new == 0) return SB_OK;
  if (!q || !o || !lse) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if ((rc = check_cache_arrays(c, n)) != SB_OK) return rc;
  const void* const buffers[] = {q, o, c->k, c->v, ws};
  if ((rc = check_aligned(buffers, 5)) != SB_OK) return rc;
  WindowParams P{};
  P.q = q; P.o = o; P.lse = lse; P.cu = n->cu_new; P.cached = n->cached; P.max_new = n->max_new;
  P.T = n->total_new; P.S = n->num_seqs; P.Hq = n->num_q_heads; P.Hkv = c->num_kv_heads; P.G = P.Hq / P.Hkv;
  P.window = window; P.sinks = sinks;
  P.scale = n->softmax_scale > 0.f ? n->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
  P.scale_log2e = P.scale * 1.4426950408889634f;
  P.cache = make_paged(c);
  const CachePlan plan = plan_cache(c, n, window, sinks);
  if (plan.few.splits > 1 || plan.many.splits > 1) {
    if (!ws) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
    P.part_o = (float*)((char*)ws + plan.part_o);
    P.part_lse = (float*)((char*)ws + plan.part_lse);
  }
  const hipStream_t st = (hipStream_t)stream;
  const bool f32 = c->dtype == SB_F32;
  const int64_t rows = P.T, seq_rows = few_seq_rows(P.G, P.max_new);
  dim3 grid, all_rows, few_rows;
  if ((rc = grid_of(plan.few.items * P.Hkv * plan.few.splits, 128, &grid)) != SB_OK || (plan.many.splits > 1 && (rc = grid_of(rows * P.Hq, 256, &all_rows)) != SB_OK) ||
      (plan.few.splits > 1 && (rc = grid_of(seq_rows * P.S * P.Hq, 256, &few_rows)) != SB_OK))
    return rc;
  KernelTimer kt(K_CACHE_ATTN, st);
  auto merge = [&](dim3 workgroups, int seq_rows) { return launch_cache_merge(P, c->head_dim, c->dtype, workgroups, seq_rows, st); };
  if (plan.many.items > 0) {
    P.splits = plan.many.splits;
    P.per_split = plan.many.per_split;
    P.part_rows = plan.many.part_rows;
    P.rows_from = f32 || plan.few.items == 0 ? 0 : kFewRows + 1;
    P.rows_to = 0x7fffffff;
    if ((rc = launch_window_fwd(P, c->head_dim, c->dtype, true, plan.many.items, st)) != SB_OK) return rc;
    if (P.splits > 1 && (rc = merge(all_rows, 0)) != SB_OK) return rc;
  }
  if (plan.few.items > 0) {
    P.splits = plan.few.splits;
    P.per_split = plan.few.per_split;
    P.part_rows = plan.few.part_rows;
    P.part_seq_rows = plan.few.part_seq_rows;
    P.rows_from = 0;
    P.rows_to = kFewRows;
    if (c->head_dim == 128) hipLaunchKernelGGL((cache_split_kernel<128>), grid, dim3(128), 0, st, P);
    else hipLaunchKernelGGL((cache_split_kernel<64>), grid, dim3(128), 0, st, P);
    SB_LAUNCH_CHECK("cache_split_kernel");
    if (P.splits > 1 && (rc = merge(few_rows, (int)seq_rows)) != SB_OK) return rc;
  }
  return SB_OK;
}

}  // extern "C"
