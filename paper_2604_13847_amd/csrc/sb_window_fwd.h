// The bfloat16 forward of window attention, for kernels whose tiles of keys and values come by different ways.
#pragma once

#include <type_traits>

#include "sb_window.h"

namespace sb {

__device__ inline f32x4 load4(const float* p) { return *(const f32x4*)p; }
__device__ inline void store4(float* p, f32x4 x) { *(f32x4*)p = x; }
__device__ inline void store4(bf16* p, f32x4 x) {
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (bf16)x[e];
  *(bf16x4*)p = y;
}

template <int D, typename T>
__device__ inline void store_column(T* to, const f32x16 (&acc)[D / 32], float f, int hf) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int vg = 0; vg < 4; ++vg)
      store4(to + 32 * dt + 8 * vg + 4 * hf, f32x4{acc[dt][4 * vg] * f, acc[dt][4 * vg + 1] * f, acc[dt][4 * vg + 2] * f, acc[dt][4 * vg + 3] * f});
}

// LSE of a row without any score above -infinity.  Over a cache it may see no key; in a packed batch it sees itself, and has no softmax: NaN, as in the block-sparse forward.
template <bool PAGED> __device__ inline float empty_lse() { return PAGED ? -__builtin_inff() : __builtin_nanf(""); }

// Pages of the tiles that come, looked up in the sequence's row of the page table (behind its end: 0) a tile before they are used.  By vector loads: waits for scalar ones are waits for LDS
// too, and all of a tile's would be waited for.
template <int D>
struct PagesAhead {
  unsigned mine;  // of this wavefront's 16 rows of the tile that is loaded next
  unsigned all;   // lane: of rows 16 (lane % 4) .. + 15 of the tile that is worked on next
  typedef KeySource<D, true> Source;
  static __device__ __attribute__((always_inline)) inline unsigned entry(const WindowParams& P, const Source& src, int u) {
    return __builtin_amdgcn_raw_buffer_load_b32(__builtin_amdgcn_make_buffer_rsrc((void*)src.pages, 0, (unsigned)P.cache.max_pages * 4, 0x20000), (u >> P.cache.page_shift) * 4, 0, 0);
  }
  __device__ __attribute__((always_inline)) inline void look_up(const WindowParams& P, const Source& src, int u) { mine = entry(P, src, u); }
  __device__ __attribute__((always_inline)) inline void look_up_all(const WindowParams& P, const Source& src, int u0, int lane) { all = entry(P, src, u0 + 16 * (lane & 3)); }
  // rows u .. u + 15, whose page is looked up: the first one's place among the pages' rows (of KV head 0), and how many exist from there on
  __device__ __attribute__((always_inline)) inline unsigned long long rows_at(const WindowParams& P, const Source& src, int u, int& rows) const {
    const unsigned p = (unsigned)__builtin_amdgcn_readfirstlane((int)mine);
    const bool any = u < src.end && (u + 16 > src.lo || u < P.sinks) && p < (unsigned)P.cache.num_pages;
    rows = any ? min(src.end - u, 16) : 0;
    return ((unsigned long long)(any ? p : 0) * P.Hkv << P.cache.page_shift) + (unsigned)(u & (P.cache.page_size - 1));
  }
  // bit x: keys u0 + 16x .. + 15 have no page.  (Those behind `end` too: where that is the page table's end, rows behind it would take them, zeros in LDS, for keys.)
  __device__ __attribute__((always_inline)) inline unsigned missing(const WindowParams& P, const Source& src, int u0, int lane) const {
    return (unsigned)__builtin_amdgcn_ballot_w64(u0 + 16 * (lane & 3) >= src.end || all >= (unsigned)P.cache.num_pages) & 15;
  }
};
struct NoPages {};

// Tiles of K and V that lie in memory as the matrix instructions take them: asynchronous loads, the next tile's while one is worked on.
template <int D, bool PAGED>
struct LoadedTiles {
  static constexpr int TILE_B = 64 * D * 2;
  RowsLoader<D, kWaves> loader;
  typename std::conditional<PAGED, PagesAhead<D>, NoPages>::type ahead;
  unsigned tiles0;
  int wave, lane;
  typedef KeySource<D, PAGED> Source;
  static_assert(64 / kWaves == 16, "a wavefront's rows of a tile lie in one page");
  __device__ inline void init(const WindowParams& P, const RowTile& t, const Source& src, int g, int wave_, int lane_, unsigned tiles0_) {
    loader.init(src.pitch, wave_, lane_);
    tiles0 = tiles0_;
    wave = wave_;
    lane = lane_;
  }
  __device__ __attribute__((always_inline)) inline void issue(const WindowParams& P, const KeyTiles<64>& keys, const Source& src, int x, int begin) const {
    const int u = 64 * keys.at(x) + 16 * wave;
    int there;
    unsigned long long o;
    if constexpr (PAGED) o = ahead.rows_at(P, src, u, there) * (D * 2);
    else o = src.rows_at(P, u, 16, there);
    const unsigned slot = tiles0 + ((x - begin) & 1) * 2 * TILE_B;
    loader.issue(src.k + o, there, slot);
    loader.issue(src.v + o, there, slot + TILE_B);
  }
  __device__ __attribute__((always_inline)) inline unsigned missing(const WindowParams& P, const KeyTiles<64>& keys, const Source& src, int x) const {
    if constexpr (PAGED) return ahead.missing(P, src, 64 * keys.at(x), lane);
    else return 0;
  }
  __device__ __attribute__((always_inline)) inline void look_up(const WindowParams& P, const KeyTiles<64>& keys, const Source& src, int x, int count) {
    if constexpr (PAGED) ahead.look_up(P, src, 64 * keys.at(min(x, count - 1)) + 16 * wave);
  }
  __device__ __attribute__((always_inline)) inline void look_up_all(const WindowParams& P, const KeyTiles<64>& keys, const Source& src, int x, int count) {
    if constexpr (PAGED) ahead.look_up_all(P, src, 64 * keys.at(min(x, count - 1)), lane);
  }
  __device__ __attribute__((always_inline)) inline void start(const WindowParams& P, const KeyTiles<64>& keys, const Source& src, int begin, int count) {
    if (begin >= count) return;
    look_up(P, keys, src, begin, count);
    issue(P, keys, src, begin, begin);
    look_up(P, keys, src, begin + 1, count);
    look_up_all(P, keys, src, begin, count);
  }
  __device__ __attribute__((always_inline)) inline void arrive(const WindowParams& P, const KeyTiles<64>& keys, const Source& src, int x, int begin, int count) {
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    if (x + 1 < count) issue(P, keys, src, x + 1, begin);
    look_up(P, keys, src, x + 2, count);
    look_up_all(P, keys, src, x + 1, count);
  }
};

// A workgroup's 32 WAVES flattened rows of KV head g, walked over tiles from .. to - 1 (those of them that there are) of their keys.  `tiles`: LDS [2][2][64 * D * 2], tile x of the walk in
// buffer (x - begin) % 2, K and V.  part: these are not all tiles that the rows see; what they add up to goes to row place(token, head, row of these) of part_o and part_lse.
template <int D, bool PAGED, int WAVES, typename Tiles, typename Params, typename Place>
__device__ __attribute__((always_inline)) inline void window_fwd_rows(const WindowParams& P, char* tiles, const Params& params, const RowTile& t, int g, int lane, int64_t from, int64_t to, bool part,
                                                                      Place place) {
  constexpr int ROWS = 32 * WAVES, ROW_B = D * 2, TILE_B = 64 * ROW_B, NOP = D / 16;
  constexpr float kLazy = 8.0f;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hf = lane >> 5;
  const int rows = t.n * P.G, mb = t.tile * ROWS, mw = mb + 32 * wave;
  auto token = [&](int m) { return (int)((unsigned)min(m, rows - 1) / (unsigned)P.G); };
  const int i = token(mw + l32), h = g * P.G + min(mw + l32, rows - 1) - i * P.G, pos = t.pos0 + i;
  // (the same in every lane, but a division leaves it in vector registers, where what the loads' resources are made of must not come from)
  auto position = [&](int m) { return __builtin_amdgcn_readfirstlane(t.pos0 + token(m)); };
  const int ta = position(mb), all_rows = position(mb + ROWS - 1), tb = PAGED ? min(all_rows, P.cache.max_pages * P.cache.page_size - 1) : all_rows;
  const int wa = position(mw), wb = position(mw + 31);  // this wavefront's
  const bool working = mw < rows;
  const KeyTiles<64> keys(ta, tb, P.window, P.sinks);
  const int begin = PAGED ? (int)min(from, (int64_t)keys.count()) : 0, count = PAGED ? (int)min(to, (int64_t)keys.count()) : keys.count();
  KeySource<D, PAGED> src;
  src.init(P, t, g, max(0, ta - P.window + 1), tb + 1);
  const unsigned tiles0 = lds_offset(tiles);
  Tiles source;
  source.init(params, t, src, g, wave, lane, tiles0);

  // B operand of S^T = K Q^T: column = row lane%32, slots = d 16ks + 8hf + (0..7)
  bf16x8 qf[NOP];
  {
    const bf16* qp = (const bf16*)P.q + ((int64_t)(t.row0 + i) * P.Hq + h) * D + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  // the query operands must have landed before the tile loads start: from here on only those are in flight, and waited for by hand
#pragma unroll
  for (int ks = 0; ks < NOP; ++ks) asm volatile("" : "+v"(qf[ks]));
  source.start(params, keys, src, begin, count);

  unsigned row_a[NOP], tr_a[D / 32][2];
#pragma unroll
  for (int ks = 0; ks < NOP; ++ks) row_a[ks] = tiles0 + l32 * ROW_B + 16 * ((2 * ks + hf) ^ chunk_swizzle<D>(l32));
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = 8 * half + 4 * hf + ((lane & 15) >> 2), d = 32 * dt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      tr_a[dt][half] = tiles0 + TILE_B + r * ROW_B + 16 * ((d >> 3) ^ chunk_swizzle<D>(r)) + 2 * (d & 7);
    }
  auto ld_row = [&](int ks, unsigned off) __attribute__((always_inline)) {
    return *(const bf16x8 __attribute__((address_space(3)))*)(uintptr_t)(row_a[ks] + off);
  };
  // A operand of O^T += V^T P^T: row = d (32dt + lane%32), slots = keys 16kk + 8(e/4) + 4hf + e%4
  auto ld_tr = [&](int kk, int dt, unsigned off) __attribute__((always_inline)) {
    const unsigned o = off + kk * 16 * ROW_B;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(tr_a[dt][0] + o));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(tr_a[dt][1] + o));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  f32x16 oacc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = zero16();
  float m = -__builtin_inff(), neg_m = 0.f, l = 0.f;
  bf16x8 op[NOP];

  auto tile = [&](auto buf_c, int u0, bool all, unsigned missing) __attribute__((always_inline)) {
    constexpr unsigned BO = decltype(buf_c)::value * 2 * TILE_B;  // the tile's buffer, as an immediate offset of every LDS read
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {  // keys 32mt .. 32mt + 31 of the tile
#pragma unroll
      for (int ks = 0; ks < NOP; ++ks) op[ks] = ld_row(ks, BO + mt * 32 * ROW_B);  // K rows
      __builtin_amdgcn_sched_barrier(0);
      f32x16 sacc = zero16();
#pragma unroll
      for (int ks = 0; ks < NOP; ++ks) {  // S^T = K Q^T, refilling every operand register with a V^T operand
        sacc = mfma32(op[ks], qf[ks], sacc);
        op[ks] = ld_tr(2 * mt + ks / (D / 32), ks % (D / 32), BO);
      }
#pragma unroll
      for (int x = 0; x < NOP; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      // max3 is inline asm, whose reads of a matrix instruction's result the compiler's hazard recogniser does not see: 12 wait states
      asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sacc));
      if (!all) {  // (one body with the mask in a branch: with a masked form of its own the accumulators were copied where the two meet)
        const Sight sees(pos, u0 + 32 * mt, hf, P.window, P.sinks);
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!sees(c_row(v, 0)) || (PAGED && (missing >> (2 * mt + (v >> 3)) & 1))) sacc[v] = -__builtin_inff();
      }
      // running maximum, followed lazily: the reference moves only when a score exceeds it by 2^kLazy
      float mx = max3(sacc[0], sacc[1], sacc[2]);
#pragma unroll
      for (int v = 3; v < 15; v += 2) mx = max3(mx, sacc[v], sacc[v + 1]);
      mx = max3(mx, sacc[15], sacc[15]);
      if (__builtin_amdgcn_ballot_w64(!((mx - m) * P.scale_log2e <= kLazy)) != 0) {
        mx = max_across_halves(mx);
        const bool first = m == -__builtin_inff();  // nothing accumulated yet for this row
        const bool move = first | ((mx - m) * P.scale_log2e > kLazy);
        const float m_new = move ? fmaxf(m, mx) : m;
        const float m_use = m_new == -__builtin_inff() ? 0.f : m_new;  // no key seen yet: keep the exponent finite
        const float alpha = first ? 1.0f : fast_exp2((m - m_use) * P.scale_log2e);
        neg_m = -m_use * P.scale_log2e;
        m = m_new;
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
          l *= alpha;
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
        }
      }
      // The sum is that of the probabilities before they are rounded to bf16 for the product with V: LSE keeps float32's precision
      bf16x8 pb[2];
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float x = fast_exp2(__builtin_fmaf(sacc[v], P.scale_log2e, neg_m));
        part[v & 3] += x;
        pb[v >> 3][v & 7] = (bf16)x;
      }
      l += (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = mfma32(op[kk * (D / 32) + dt], pb[kk], oacc[dt]);
    }
  };
  auto visit = [&](auto buf_c, int x) __attribute__((always_inline)) {
    const int u0 = 64 * keys.at(x);
    const unsigned missing = source.missing(params, keys, src, x);
    source.arrive(params, keys, src, x, begin, count);  // tile x is there for everyone; everyone is done with tile x - 1
    const bool none = !working || u0 > wb || (wa - (u0 + 63) >= P.window && u0 >= P.sinks);
    const bool all = u0 + 63 <= wa && (wb - u0 < P.window || u0 + 63 < P.sinks) && missing == 0;
    if (!none) tile(buf_c, u0, all, missing);
  };
  int x = begin;
  for (; x + 2 <= count; x += 2) {  // two tiles a turn, so that a tile's buffer is known at compile time
    visit(std::integral_constant<int, 0>(), x);
    visit(std::integral_constant<int, 1>(), x + 1);
  }
  if (x < count) visit(std::integral_constant<int, 0>(), x);
  wait_vmcnt<0>();

  l += __shfl_xor(l, 32, 64);  // the two lane halves hold different keys of the same row
  // (a sum that is no number is not one that saw nothing; in a packed batch a sum of zero makes O what it makes LSE: 0 / 0)
  const float inv = PAGED && l == 0.f ? 0.f : 1.0f / l;
  if (PAGED && part) {
    if (mw + l32 >= rows) return;
    const int64_t row = place(i, h, 32 * wave + l32);
    if (hf == 0) P.part_lse[row] = l == 0.f ? -__builtin_inff() : m * P.scale_log2e + __builtin_log2f(l);
    if (l != 0.f) store_column<D>(P.part_o + row * D, oacc, inv, hf);
    return;
  }
  __syncthreads();  // the tiles' LDS is free
  store_tile<D>(tiles + wave * 32 * ROW_B, lane, [&](int dt, int v) __attribute__((always_inline)) { return oacc[dt][v] * inv; },
                [&](int r) __attribute__((always_inline)) -> bf16* {
                  if (mw + r >= rows) return nullptr;
                  const int j = token(mw + r);
                  return (bf16*)P.o + ((int64_t)(t.row0 + j) * P.Hq + g * P.G + mw + r - j * P.G) * D;
                });
  if (hf == 0 && mw + l32 < rows)
    P.lse[(int64_t)h * P.T + t.row0 + i] = l == 0.f ? empty_lse<PAGED>() : (m * P.scale_log2e + __builtin_log2f(l)) * 0.69314718055994531f;
}

}  // namespace sb
