// Attention with a sliding window and sinks, forward and backward, over packed batches or (forward) over a paged cache.
//
//   S = scale Q K^T,  row t sees u <= t with t - u < window or u < sinks,  P = softmax(S),  O = P V,  LSE = log sum exp S
//   Dr = rowsum(dO * O),  dP = dO V^T,  dS = P * (dP - Dr),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// All products are computed with the query (forward, dQ) or the key (dK/dV) in a column of the matrix instructions' result, as S^T = K Q^T: statistics are then
// per lane, and a result is the next product's operand without any cross-lane movement (c_row).
#include <math.h>

#include <type_traits>

#include "sb_window.h"

namespace sb {

// ---------------------------------------------------------------------------------------------
// float32 arithmetic throughout: v_mfma_f32_32x32x2_f32, operands straight from memory.  One wavefront owns 32 rows (or 32 keys)
// and walks strips of 32 keys (rows).  Operand layout per lane: A row / B column = lane%32, contraction slot = lane/32.
__device__ inline f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

__device__ inline f32x4 load4(const float* p) { return *(const f32x4*)p; }
__device__ inline f32x4 load4(const bf16* p) {
  const bf16x4 x = *(const bf16x4*)p;
  return f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
}
__device__ inline void store4(float* p, f32x4 x) { *(f32x4*)p = x; }
__device__ inline void store4(bf16* p, f32x4 x) {
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (bf16)x[e];
  *(bf16x4*)p = y;
}

// A row of D elements as an operand of a product over d: step x covers d = 8x .. 8x + 7, four instructions with slot hf at 8x + 4hf + j.
template <int D> struct RowOperand { f32x4 x[D / 8]; };
template <int D, typename T>
__device__ inline void load_row(RowOperand<D>& r, const T* row, int hf) {
#pragma unroll
  for (int x = 0; x < D / 8; ++x) r.x[x] = row ? load4(row + 8 * x + 4 * hf) : f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int D>
__device__ inline f32x16 dot_rows(const RowOperand<D>& a, const RowOperand<D>& b) {
  f32x16 s = zero16();
#pragma unroll
  for (int x = 0; x < D / 8; ++x)
#pragma unroll
    for (int j = 0; j < 4; ++j) s = mfma_f32(a.x[x][j], b.x[x][j], s);
  return s;
}
// acc[dt] += X^T w over 32 rows of X, row c_row(v, hf) with weight w[v]; row(r) is a row's address or null
template <int D, typename T, typename F>
__device__ inline void add_rows(f32x16 (&acc)[D / 32], const float (&w)[16], int l32, int hf, F row) {
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const T* x = row(c_row(v, hf));
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) acc[dt] = mfma_f32(x ? (float)x[32 * dt + l32] : 0.f, w[v], acc[dt]);
  }
}
template <int D, typename T>
__device__ inline void store_column(T* to, const f32x16 (&acc)[D / 32], float f, int hf) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int vg = 0; vg < 4; ++vg)
      store4(to + 32 * dt + 8 * vg + 4 * hf, f32x4{acc[dt][4 * vg] * f, acc[dt][4 * vg + 1] * f, acc[dt][4 * vg + 2] * f, acc[dt][4 * vg + 3] * f});
}

// Keys that no row of the wavefront sees (behind the last row, between the sinks and the window) are not read: their weights are zero, but what they hold
// may be no number.
template <typename T, int D, bool PAGED>
struct Keys {
  const WindowParams& P;
  const RowTile& t;
  int g, lo, hi;  // seen: u < sinks or lo <= u < hi
  __device__ inline int64_t offset(int u) const {
    if (u >= hi || (u < lo && u >= P.sinks)) return -1;
    if (PAGED) {
      const int64_t r = P.cache.row_of(t.s, u, g);
      return r < 0 ? -1 : r * D;
    }
    return ((int64_t)(t.row0 + u) * P.Hkv + g) * D;
  }
  __device__ inline const T* k(int u) const { const int64_t o = offset(u); return o < 0 ? nullptr : (const T*)(PAGED ? P.cache.k : P.k) + o; }
  __device__ inline const T* v(int u) const { const int64_t o = offset(u); return o < 0 ? nullptr : (const T*)(PAGED ? P.cache.v : P.v) + o; }
};

template <typename T, int D, bool PAGED>
__global__ __launch_bounds__(256) void window_fwd_f32_kernel(WindowParams P, int64_t items) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  if (item >= items) return;
  const RowTile t = locate_tile<32, PAGED>(P, item / P.Hkv);
  if (t.s < 0) return;
  const int g = (int)(item % P.Hkv);
  const int64_t rows = (int64_t)t.n * P.G, m0 = (int64_t)t.tile * 32, m = min(m0 + l32, rows - 1);
  const int i = (int)(m / P.G), h = g * P.G + (int)(m % P.G);
  const int ta = t.pos0 + (int)(m0 / P.G), tb = t.pos0 + (int)(min(m0 + 31, rows - 1) / P.G), pos = t.pos0 + i;
  const int64_t at = ((int64_t)(t.row0 + i) * P.Hq + h) * D;
  RowOperand<D> qr, kr;
  load_row<D>(qr, (const T*)P.q + at, hf);
  const int last = PAGED ? min(tb, P.cache.max_pages * P.cache.page_size - 1) : tb;
  const KeyTiles<32> tiles(ta, last, P.window, P.sinks);
  const Keys<T, D, PAGED> keys{P, t, g, max(0, ta - P.window + 1), last + 1};
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  float top = -__builtin_inff(), l = 0.f;  // largest score seen (in units of log 2), sum of exponentials
  for (int x = 0; x < tiles.count(); ++x) {
    const int u0 = 32 * tiles.at(x);
    const T* kp = keys.k(u0 + l32);
    load_row<D>(kr, kp, hf);
    f32x16 sc = dot_rows<D>(kr, qr);
    const unsigned exists = (unsigned)__builtin_amdgcn_ballot_w64(kp != nullptr);
    float mx = -__builtin_inff(), p[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = c_row(v, hf);
      p[v] = sees(pos, u0 + r, P.window, P.sinks) && (exists >> r & 1) ? sc[v] * P.scale_log2e : -__builtin_inff();
      mx = fmaxf(mx, p[v]);
    }
    mx = fmaxf(top, max_across_halves(mx));
    const float ref = mx == -__builtin_inff() ? 0.f : mx;  // nothing seen yet: keep the exponents finite
    const float alpha = fast_exp2(top - ref);
    top = mx;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[dt][v] *= alpha;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v] = fast_exp2(p[v] - ref);
      l += p[v];
    }
    add_rows<D, T>(acc, p, l32, hf, [&](int r) { return keys.v(u0 + r); });
  }
  l += __shfl_xor(l, 32, 64);
  if (m0 + l32 >= rows) return;
  store_column<D>((T*)P.o + at, acc, l == 0.f ? 0.f : 1.0f / l, hf);
  if (hf == 0) P.lse[(int64_t)h * P.T + t.row0 + i] = l == 0.f ? -__builtin_inff() : (top + __builtin_log2f(l)) * 0.69314718055994531f;
}

// Dr = rowsum(dO * O), one wavefront per row: 16 or 32 lanes each hold four elements.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_delta_kernel(WindowParams P, int64_t rows) {
  constexpr int LANES = D / 4, PER = 256 / LANES;
  const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;
  const int c = threadIdx.x % LANES;
  float x = 0.f;
  if (row < rows) {
    const f32x4 a = load4((const T*)P.o_in + row * D + 4 * c), b = load4((const T*)P.d_o + row * D + 4 * c);
    x = a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3];
  }
#pragma unroll
  for (int off = LANES / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  if (row < rows && c == 0) P.delta[row % P.Hq * P.T + row / P.Hq] = x;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void window_dq_f32_kernel(WindowParams P, int64_t items) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  if (item >= items) return;
  const RowTile t = locate_tile<32, false>(P, item / P.Hkv);
  if (t.s < 0) return;
  const int g = (int)(item % P.Hkv);
  const int64_t rows = (int64_t)t.n * P.G, m0 = (int64_t)t.tile * 32, m = min(m0 + l32, rows - 1);
  const int i = (int)(m / P.G), h = g * P.G + (int)(m % P.G);
  const int ta = (int)(m0 / P.G), tb = (int)(min(m0 + 31, rows - 1) / P.G);
  const int64_t at = ((int64_t)(t.row0 + i) * P.Hq + h) * D;
  RowOperand<D> qr, dor, x;
  load_row<D>(qr, (const T*)P.q + at, hf);
  load_row<D>(dor, (const T*)P.d_o + at, hf);
  const float lse2 = P.lse[(int64_t)h * P.T + t.row0 + i] * 1.4426950408889634f, dr = P.delta[(int64_t)h * P.T + t.row0 + i];
  const KeyTiles<32> tiles(ta, tb, P.window, P.sinks);
  const Keys<T, D, false> keys{P, t, g, max(0, ta - P.window + 1), tb + 1};
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  for (int y = 0; y < tiles.count(); ++y) {
    const int u0 = 32 * tiles.at(y);
    load_row<D>(x, keys.k(u0 + l32), hf);
    const f32x16 sc = dot_rows<D>(x, qr);
    load_row<D>(x, keys.v(u0 + l32), hf);
    const f32x16 dp = dot_rows<D>(x, dor);
    float ds[16];
#pragma unroll
    for (int v = 0; v < 16; ++v)
      ds[v] = sees(i, u0 + c_row(v, hf), P.window, P.sinks) ? fast_exp2(__builtin_fmaf(sc[v], P.scale_log2e, -lse2)) * (dp[v] - dr) : 0.f;
    add_rows<D, T>(acc, ds, l32, hf, [&](int r) { return keys.k(u0 + r); });
  }
  if (m0 + l32 < rows) store_column<D>((T*)P.dq + at, acc, P.scale, hf);
}

// Key-major: one wavefront owns 32 keys of a KV head and walks the flattened rows that see any of them, 32 at a time, in order.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_dkv_f32_kernel(WindowParams P, int64_t items) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  if (item >= items) return;
  WindowParams one = P;  // tiles of 32 keys: one "row" a token
  one.G = 1;
  const RowTile t = locate_tile<32, false>(one, item / P.Hkv);
  if (t.s < 0) return;
  const int g = (int)(item % P.Hkv);
  const int u0 = t.tile * 32, u = min(u0 + l32, t.n - 1), last = min(u0 + 31, t.n - 1);
  const int64_t at = ((int64_t)(t.row0 + u) * P.Hkv + g) * D;
  RowOperand<D> kr, vr, x;
  load_row<D>(kr, (const T*)P.k + at, hf);
  load_row<D>(vr, (const T*)P.v + at, hf);
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) dk[dt] = dv[dt] = zero16();
  const int64_t behind = u0 < P.sinks ? t.n : min((int64_t)t.n, (int64_t)last + P.window);  // the first token that sees none of them
  const int64_t end = behind * P.G;
  auto row = [&](int64_t m) { return ((int64_t)(t.row0 + (int)(m / P.G)) * P.Hq + g * P.G + (int)(m % P.G)) * D; };
  for (int64_t m0 = (int64_t)u0 * P.G; m0 < end; m0 += 32) {
    const bool there = m0 + l32 < end;
    load_row<D>(x, there ? (const T*)P.q + row(m0 + l32) : nullptr, hf);
    const f32x16 sc = dot_rows<D>(x, kr);
    load_row<D>(x, there ? (const T*)P.d_o + row(m0 + l32) : nullptr, hf);
    const f32x16 dp = dot_rows<D>(x, vr);
    // statistics of row m0 + lane%32, passed on to the lanes that hold the row
    const int64_t m = there ? m0 + l32 : end - 1;
    const int64_t stat = (int64_t)(g * P.G + (int)(m % P.G)) * P.T + t.row0 + (int)(m / P.G);
    const float lse2 = P.lse[stat] * 1.4426950408889634f, dr = P.delta[stat];
    const int pos = there ? (int)(m / P.G) : -1;
    float p[16], ds[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int r = c_row(v, hf);
      const float e = __shfl(lse2, r, 64), d = __shfl(dr, r, 64);
      const int tr = __shfl(pos, r, 64);
      const bool seen = tr >= 0 && sees(tr, u, P.window, P.sinks);
      p[v] = seen ? fast_exp2(__builtin_fmaf(sc[v], P.scale_log2e, -e)) : 0.f;
      ds[v] = seen ? p[v] * (dp[v] - d) : 0.f;
    }
    add_rows<D, T>(dv, p, l32, hf, [&](int r) { return m0 + r < end ? (const T*)P.d_o + row(m0 + r) : nullptr; });
    add_rows<D, T>(dk, ds, l32, hf, [&](int r) { return m0 + r < end ? (const T*)P.q + row(m0 + r) : nullptr; });
  }
  if (u0 + l32 < t.n) {
    store_column<D>((T*)P.dk + at, dk, P.scale, hf);
    store_column<D>((T*)P.dv + at, dv, 1.0f, hf);
  }
}

// ---------------------------------------------------------------------------------------------
// bfloat16 forward.  A workgroup of eight wavefronts owns 256 flattened rows of a KV head, 32 a wavefront, and walks the 64-key tiles that any of them sees; K and V tiles are
// shared in LDS and double-buffered by asynchronous loads.  A wavefront takes a tile as two halves of 32 keys, a step of the running softmax each.  A tile that a wavefront's rows
// all see carries no mask; one that none of them sees is only waited for.  256 registers, so two wavefronts share a SIMD: one runs its exponentials while the other runs matrix
// instructions.
template <int D, bool PAGED>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void window_fwd_kernel(WindowParams P) {
  constexpr int ROWS = 256, ROW_B = D * 2, TILE_B = 64 * ROW_B, NOP = D / 16;
  constexpr float kLazy = 8.0f;
  __shared__ __attribute__((aligned(1024))) char tiles[2][2][TILE_B];  // [buffer][K, V]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const RowTile t = locate_tile<ROWS, PAGED>(P, blockIdx.x / P.Hkv);
  if (t.s < 0) return;
  const int g = (int)(blockIdx.x % P.Hkv);
  const int64_t rows = (int64_t)t.n * P.G, mb = (int64_t)t.tile * ROWS, mw = mb + 32 * wave;
  auto token = [&](int64_t m) { return (int)(min(m, rows - 1) / P.G); };
  const int i = token(mw + l32), h = g * P.G + (int)(min(mw + l32, rows - 1) - (int64_t)i * P.G), pos = t.pos0 + i;
  const int ta = t.pos0 + token(mb);
  const int tb = PAGED ? min(t.pos0 + token(mb + ROWS - 1), P.cache.max_pages * P.cache.page_size - 1) : token(mb + ROWS - 1);
  const int wa = t.pos0 + token(mw), wb = t.pos0 + token(mw + 31);  // this wavefront's
  const bool working = mw < rows;
  const KeyTiles<64> keys(ta, tb, P.window, P.sinks);
  const int count = keys.count();
  KeySource<D, PAGED> src;
  src.init(P, t, g, max(0, ta - P.window + 1), tb + 1);
  RowsLoader<D> loader;
  loader.init(src.pitch, wave, lane);
  const unsigned tiles0 = lds_offset(&tiles[0][0][0]);
  auto issue = [&](int x) {
    const int u = 64 * keys.at(x) + 8 * wave;
    int there;
    const unsigned long long o = src.rows_at(P, u, 8, there);
    const unsigned slot = tiles0 + (x & 1) * 2 * TILE_B;
    loader.issue(src.k + o, there, slot);
    loader.issue(src.v + o, there, slot + TILE_B);
  };

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
  issue(0);

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

  auto tile = [&](auto mask_c, auto buf_c, int u0, unsigned missing) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mask_c)::value;
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
      if (MASK) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 32 * mt + c_row(v, hf);
          if (!sees(pos, u0 + r, P.window, P.sinks) || (PAGED && (missing >> (r >> 4) & 1))) sacc[v] = -__builtin_inff();
        }
      } else {
        // max3 is inline asm, whose reads of a matrix instruction's result the compiler's hazard recogniser does not see: 12 wait states
        asm volatile("s_nop 7\n\ts_nop 3" : "+v"(sacc));
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
    const unsigned missing = src.missing(P, u0);
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();  // tile x has landed for everyone; everyone is done with tile x - 1
    if (x + 1 < count) issue(x + 1);
    const bool none = !working || u0 > wb || (wa - (u0 + 63) >= P.window && u0 >= P.sinks);
    const bool all = u0 + 63 <= wa && (wb - u0 < P.window || u0 + 63 < P.sinks) && missing == 0;
    if (none) return;
    if (all) tile(std::false_type(), buf_c, u0, 0u);
    else tile(std::true_type(), buf_c, u0, missing);
  };
  int x = 0;
  for (; x + 2 <= count; x += 2) {  // two tiles a turn, so that a tile's buffer is known at compile time
    visit(std::integral_constant<int, 0>(), x);
    visit(std::integral_constant<int, 1>(), x + 1);
  }
  if (x < count) visit(std::integral_constant<int, 0>(), x);
  wait_vmcnt<0>();

  l += __shfl_xor(l, 32, 64);  // the two lane halves hold different keys of the same row
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  __syncthreads();  // the tiles' LDS is free
  store_tile<D>(&tiles[0][0][0] + wave * 32 * ROW_B, lane, [&](int dt, int v) __attribute__((always_inline)) { return oacc[dt][v] * inv; },
                [&](int r) __attribute__((always_inline)) -> bf16* {
                  if (mw + r >= rows) return nullptr;
                  const int j = token(mw + r);
                  return (bf16*)P.o + ((int64_t)(t.row0 + j) * P.Hq + g * P.G + (int)(mw + r - (int64_t)j * P.G)) * D;
                });
  if (hf == 0 && mw + l32 < rows)
    P.lse[(int64_t)h * P.T + t.row0 + i] = l > 0.f ? (m * P.scale_log2e + __builtin_log2f(l)) * 0.69314718055994531f : -__builtin_inff();
}

// ---------------------------------------------------------------------------------------------
int64_t row_tiles(const int32_t* cu, int S, int G, int rows) {
  int64_t n = 0;
  for (int s = 0; s < S; ++s) n += ((int64_t)(cu[s + 1] - cu[s]) * G + rows - 1) / rows;
  return n;
}
int64_t row_tiles_most(int total, int S, int G, int rows) { return ((int64_t)total * G) / rows + S; }

template <typename F>
static int with_types(int D, int dtype, F f) {
  if (dtype == SB_F32) return D == 128 ? f(float(), std::integral_constant<int, 128>()) : f(float(), std::integral_constant<int, 64>());
  return D == 128 ? f(bf16(), std::integral_constant<int, 128>()) : f(bf16(), std::integral_constant<int, 64>());
}
static int grid_of(int64_t workgroups, dim3* grid) {
  if (workgroups > 0x3fffffll) { set_error("too many tiles for one launch"); return SB_ERR_UNSUPPORTED; }
  *grid = dim3((unsigned)workgroups);
  return SB_OK;
}

int launch_window_fwd(const WindowParams& P, int D, int dtype, bool paged, int64_t tiles, hipStream_t st) {
  const int64_t items = tiles * P.Hkv;
  dim3 grid;
  const int rc = grid_of(dtype == SB_F32 ? (items + 3) / 4 : items, &grid);
  if (rc != SB_OK) return rc;
  auto launch = [&](auto d, auto pg) {
    constexpr int DD = decltype(d)::value;
    constexpr bool PAGED = decltype(pg)::value;
    if (dtype == SB_F32) hipLaunchKernelGGL((window_fwd_f32_kernel<float, DD, PAGED>), grid, dim3(256), 0, st, P, items);
    else hipLaunchKernelGGL((window_fwd_kernel<DD, PAGED>), grid, dim3(512), 0, st, P);
  };
  auto with_d = [&](auto pg) { if (D == 128) launch(std::integral_constant<int, 128>(), pg); else launch(std::integral_constant<int, 64>(), pg); };
  if (paged) with_d(std::true_type()); else with_d(std::false_type());
  SB_LAUNCH_CHECK("window_fwd_kernel");
  return SB_OK;
}

static int check_window(const sb_problem* p, int32_t window, int32_t sinks, Geo* g) {
  const int rc = make_batch(p, g);
  if (rc != SB_OK) return rc;
  if (window < 1 || sinks < 0) { set_error("window (%d) must be at least 1 and sinks (%d) not negative", window, sinks); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}
static WindowParams window_params(const Geo& g, const sb_problem* p, int32_t window, int32_t sinks) {
  WindowParams P{};
  P.cu = p->cu_seqlens_dev;
  P.T = g.T; P.S = g.S; P.Hq = g.Hq; P.Hkv = g.Hkv; P.G = g.G;
  P.window = window; P.sinks = sinks;
  P.scale = g.softmax_scale; P.scale_log2e = g.softmax_scale * 1.4426950408889634f;
  return P;
}

struct WindowWs { size_t delta, bytes; };
static WindowWs window_bwd_ws(const Geo& g) {
  WindowWs w{};
  size_t o = 0;
  w.delta = o; o = align_up(o + sizeof(float) * (size_t)g.T * g.Hq);
  w.bytes = o;
  return w;
}

}  // namespace sb

using namespace sb;

extern "C" {

int sb_window_ws_bytes(const sb_problem* p, int32_t window, int32_t sinks, int64_t* fwd_bytes, int64_t* bwd_bytes) {
  Geo g;
  const int rc = check_window(p, window, sinks, &g);
  if (rc != SB_OK) return rc;
  if (fwd_bytes) *fwd_bytes = 0;
  if (bwd_bytes) *bwd_bytes = (int64_t)window_bwd_ws(g).bytes;
  return SB_OK;
}

int sb_window_attn_fwd(const sb_problem* p, int32_t window, int32_t sinks, const void* q, const void* k, const void* v, void* o, float* lse, void* ws,
                       void* stream) {
  Geo g;
  const int rc = check_window(p, window, sinks, &g);
  if (rc != SB_OK) return rc;
  if (g.T == 0) return SB_OK;
  if (!p->cu_seqlens_dev) { set_error("cu_seqlens_dev is required"); return SB_ERR_INVALID_ARG; }
  if (!q || !k || !v || !o || !lse) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  WindowParams P = window_params(g, p, window, sinks);
  P.q = q; P.k = k; P.v = v; P.o = o; P.lse = lse;
  KernelTimer kt(K_WINDOW_FWD, (hipStream_t)stream);
  return launch_window_fwd(P, g.D, g.dtype, false, row_tiles(p->cu_seqlens_host, g.S, g.G, forward_rows(g.dtype)), (hipStream_t)stream);
}

int sb_window_attn_bwd(const sb_problem* p, int32_t window, int32_t sinks, const void* q, const void* k, const void* v, const void* o,
                       const float* lse, const void* d_o, void* dq, void* dk, void* dv, void* ws, void* stream) {
  Geo g;
  int rc = check_window(p, window, sinks, &g);
  if (rc != SB_OK) return rc;
  if (g.T == 0) return SB_OK;
  if (!p->cu_seqlens_dev) { set_error("cu_seqlens_dev is required"); return SB_ERR_INVALID_ARG; }
  if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv || !ws) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  const hipStream_t st = (hipStream_t)stream;
  WindowParams P = window_params(g, p, window, sinks);
  P.q = q; P.k = k; P.v = v; P.o_in = o; P.lse = (float*)lse; P.d_o = d_o; P.dq = dq; P.dk = dk; P.dv = dv;
  P.delta = (float*)((char*)ws + window_bwd_ws(g).delta);
  const int64_t rows = (int64_t)g.T * g.Hq, per = 1024 / g.D;
  const int64_t q_items = row_tiles(p->cu_seqlens_host, g.S, g.G, 32) * g.Hkv, k_items = row_tiles(p->cu_seqlens_host, g.S, 1, 32) * g.Hkv;
  dim3 delta_grid, q_grid, k_grid;
  if ((rc = grid_of((rows + per - 1) / per, &delta_grid)) != SB_OK || (rc = grid_of((q_items + 3) / 4, &q_grid)) != SB_OK ||
      (rc = grid_of((k_items + 3) / 4, &k_grid)) != SB_OK)
    return rc;
  return with_types(g.D, g.dtype, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int DD = decltype(d)::value;
    {
      KernelTimer kt(K_WINDOW_DQ, st);
      hipLaunchKernelGGL((window_delta_kernel<T, DD>), delta_grid, dim3(256), 0, st, P, rows);
      SB_LAUNCH_CHECK("window_delta_kernel");
      hipLaunchKernelGGL((window_dq_f32_kernel<T, DD>), q_grid, dim3(256), 0, st, P, q_items);
      SB_LAUNCH_CHECK("window_dq_f32_kernel");
    }
    KernelTimer kt(K_WINDOW_DKV, st);
    hipLaunchKernelGGL((window_dkv_f32_kernel<T, DD>), k_grid, dim3(256), 0, st, P, k_items);
    SB_LAUNCH_CHECK("window_dkv_f32_kernel");
    return SB_OK;
  });
}

}  // extern "C"
