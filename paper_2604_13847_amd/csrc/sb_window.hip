// Attention with a sliding window and sinks, forward and backward, over packed batches or (forward) over a paged cache.
//
//   S = scale Q K^T,  row t sees u <= t with t - u < window or u < sinks,  P = softmax(S),  O = P V,  LSE = log sum exp S
//   Dr = rowsum(dO * O),  dP = dO V^T,  dS = P * (dP - Dr),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// All products are computed with the query (forward, dQ) or the key (dK/dV) in a column of the matrix instructions' result, as S^T = K Q^T: statistics are then
// per lane, and a result is the next product's operand without any cross-lane movement (c_row).
#include <math.h>

#include <type_traits>

#include "sb_window_fwd.h"

namespace sb {

// ---------------------------------------------------------------------------------------------
// float32 arithmetic throughout: v_mfma_f32_32x32x2_f32, operands straight from memory.  A workgroup owns 32 rows (or 32 keys) and walks strips of 32 keys (rows), in
// turn to its wavefronts; the wavefronts' sums are added in order at the end.  Operand layout per lane: A row / B column = lane%32, contraction slot = lane/32.
__device__ inline f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// A row of D elements as an operand of a product over d: step x covers d = 8x .. 8x + 7, four instructions with slot hf at 8x + 4hf + j.
template <int D> struct RowOperand { f32x4 x[D / 8]; };
// A row that is null counts as zeros; `any`, some row that may be read, stands in for it, so that no load is behind a branch and all are on their way together.
template <int D, typename T>
__device__ inline void load_row(RowOperand<D>& r, const T* row, const T* any, int hf) {
  const T* const from = row ? row : any;
#pragma unroll
  for (int x = 0; x < D / 8; ++x) r.x[x] = load4(from + 8 * x + 4 * hf);
  if (!row) {
#pragma unroll
    for (int x = 0; x < D / 8; ++x) r.x[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
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
template <int D>
__device__ inline f32x16 dot_rows(const RowOperand<D>& a, const f32x4 (&b)[D / 8][64], int lane) {
  f32x16 s = zero16();
#pragma unroll
  for (int x = 0; x < D / 8; ++x) {
    const f32x4 y = b[x][lane];
#pragma unroll
    for (int j = 0; j < 4; ++j) s = mfma_f32(a.x[x][j], y[j], s);
  }
  return s;
}
// acc[dt] += X^T w over 32 rows of X, row c_row(v, hf) with weight w[v]; row(r) is a row's address or null
template <int D, typename T, typename F>
__device__ inline void add_rows(f32x16 (&acc)[D / 32], const float (&w)[16], const T* any, int l32, int hf, F row) {
#pragma unroll
  for (int v0 = 0; v0 < 16; v0 += 8) {
    T x[8][D / 32];
    bool there[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      const T* const r = row(c_row(v0 + v, hf));
      there[v] = r != nullptr;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) x[v][dt] = (r ? r : any)[32 * dt + l32];
    }
#pragma unroll
    for (int v = 0; v < 8; ++v)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) acc[dt] = mfma_f32(there[v] ? (float)x[v][dt] : 0.f, w[v0 + v], acc[dt]);
  }
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

// The other wavefronts' registers for the first one
template <int N, int W>
struct Sums {
  float x[W - 1][N][64];
  __device__ inline void put(int wave, int i, int lane, float v) { if (wave > 0) x[wave - 1][i][lane] = v; }
};

template <typename T, int D, bool PAGED>
__global__ __launch_bounds__(256) void window_fwd_f32_kernel(WindowParams P) {
  constexpr int NR = 16 * (D / 32);
  __shared__ Sums<NR + 2, 4> sums;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const unsigned item = blockIdx.x;
  const int splits = PAGED ? P.splits : 1, z = (int)(item / P.Hkv % splits);
  const RowTile t = locate_tile<32, PAGED>(P, item / P.Hkv / splits);
  if (t.s < 0) return;
  const int g = (int)(item % P.Hkv);
  const int64_t rows = (int64_t)t.n * P.G, m0 = (int64_t)t.tile * 32, m = min(m0 + l32, rows - 1);
  const int i = (int)(m / P.G), h = g * P.G + (int)(m % P.G);
  const int ta = t.pos0 + (int)(m0 / P.G), tb = t.pos0 + (int)(min(m0 + 31, rows - 1) / P.G), pos = t.pos0 + i;
  const int64_t at = ((int64_t)(t.row0 + i) * P.Hq + h) * D;
  RowOperand<D> qr, kr;
  const T* const any = (const T*)P.q + at;
  load_row<D>(qr, any, any, hf);
  const int last = PAGED ? min(tb, P.cache.max_pages * P.cache.page_size - 1) : tb;
  const KeyTiles<32> tiles(ta, last, P.window, P.sinks);
  const Keys<T, D, PAGED> keys{P, t, g, max(0, ta - P.window + 1), last + 1};
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  float top = -__builtin_inff(), l = 0.f;  // largest score seen (in units of log 2), sum of exponentials
  const int x0 = PAGED ? (int)min((int64_t)z * P.per_split, (int64_t)tiles.count()) : 0;
  const int x1 = PAGED && z < splits - 1 ? min(x0 + P.per_split, tiles.count()) : tiles.count();
  for (int x = x0 + wave; x < x1; x += 4) {
    const int u0 = 32 * tiles.at(x);
    const T* kp = keys.k(u0 + l32);
    load_row<D>(kr, kp, any, hf);
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
    add_rows<D, T>(acc, p, any, l32, hf, [&](int r) { return keys.v(u0 + r); });
  }
  l += __shfl_xor(l, 32, 64);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) sums.put(wave, 16 * dt + v, lane, acc[dt][v]);
  sums.put(wave, NR, lane, top);
  sums.put(wave, NR + 1, lane, l);
  __syncthreads();
  if (wave > 0) return;
  float best = top;
#pragma unroll
  for (int w = 0; w < 3; ++w) best = fmaxf(best, sums.x[w][NR][lane]);
  const float ref = best == -__builtin_inff() ? 0.f : best, f0 = fast_exp2(top - ref);
  l *= f0;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] *= f0;
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const float f = fast_exp2(sums.x[w][NR][lane] - ref);
    l += f * sums.x[w][NR + 1][lane];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[dt][v] = __builtin_fmaf(f, sums.x[w][16 * dt + v][lane], acc[dt][v]);
  }
  top = best;
  if (m0 + l32 >= rows) return;
  if (splits > 1) {
    if (l != 0.f) store_column<D>(P.part_o + (int64_t)z * P.T * P.Hq * D + at, acc, 1.0f / l, hf);
    if (hf == 0) P.part_lse[(int64_t)z * P.T * P.Hq + at / D] = l == 0.f ? -__builtin_inff() : top + __builtin_log2f(l);
    return;
  }
  store_column<D>((T*)P.o + at, acc, PAGED && l == 0.f ? 0.f : 1.0f / l, hf);  // (see the bfloat16 kernel)
  if (hf == 0) P.lse[(int64_t)h * P.T + t.row0 + i] = l == 0.f ? empty_lse<PAGED>() : (top + __builtin_log2f(l)) * 0.69314718055994531f;
}

// Dr = rowsum(dO * O): 16 or 32 lanes to a row, four elements each.  (bfloat16: the dQ kernel does this.)
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
  if (row < rows && c == 0) {
    P.dr[row] = x;
    P.lse2[row] = P.lse[row % P.Hq * P.T + row / P.Hq] * 1.4426950408889634f;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void window_dq_f32_kernel(WindowParams P) {
  __shared__ Sums<16 * (D / 32), 4> sums;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const unsigned item = blockIdx.x;
  const RowTile t = locate_tile<32, false>(P, item / P.Hkv);
  if (t.s < 0) return;
  const int g = (int)(item % P.Hkv);
  const int64_t rows = (int64_t)t.n * P.G, m0 = (int64_t)t.tile * 32, m = min(m0 + l32, rows - 1);
  const int i = (int)(m / P.G), h = g * P.G + (int)(m % P.G);
  const int ta = (int)(m0 / P.G), tb = (int)(min(m0 + 31, rows - 1) / P.G);
  const int64_t at = ((int64_t)(t.row0 + i) * P.Hq + h) * D;
  RowOperand<D> qr, dor, x;
  const T* const any = (const T*)P.q + at;
  load_row<D>(qr, any, any, hf);
  load_row<D>(dor, (const T*)P.d_o + at, any, hf);
  const float lse2 = P.lse2[at / D], dr = P.dr[at / D];
  const KeyTiles<32> tiles(ta, tb, P.window, P.sinks);
  const Keys<T, D, false> keys{P, t, g, max(0, ta - P.window + 1), tb + 1};
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  for (int y = wave; y < tiles.count(); y += 4) {
    const int u0 = 32 * tiles.at(y);
    load_row<D>(x, keys.k(u0 + l32), any, hf);
    const f32x16 sc = dot_rows<D>(x, qr);
    load_row<D>(x, keys.v(u0 + l32), any, hf);
    const f32x16 dp = dot_rows<D>(x, dor);
    float ds[16];
#pragma unroll
    for (int v = 0; v < 16; ++v)
      ds[v] = sees(i, u0 + c_row(v, hf), P.window, P.sinks) ? fast_exp2(__builtin_fmaf(sc[v], P.scale_log2e, -lse2)) * (dp[v] - dr) : 0.f;
    add_rows<D, T>(acc, ds, any, l32, hf, [&](int r) { return keys.k(u0 + r); });
  }
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) sums.put(wave, 16 * dt + v, lane, acc[dt][v]);
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[dt][v] += sums.x[w][16 * dt + v][lane];
  if (m0 + l32 < rows) store_column<D>((T*)P.dq + at, acc, P.scale, hf);
}

// Key-major: a workgroup owns 32 keys of a KV head and walks the flattened rows that see any of them, 32 at a time, in turn to its wavefronts; their sums are added in order.  At
// head_dim 64 two wavefronts share a SIMD, each with 256 registers (16384 tokens, 8/2 heads, window 1024, 4 sinks: 5.4 ms with one, 4.2 with two); at 128 the sums alone take 256.
// Sinks have no items of their own here: their tile's workgroup walks all rows of its sequence, and the launch is as long as that (the same without sinks: 1.0 ms).
// PARTS: where items are few, near_parts workgroups share the rows of one, and window_dkv_f32_join_kernel adds their sums in order.  1024 tokens, one head, head_dim 64, window 200,
// 4 sinks: 60 us whole (four wavefronts 72), 26 in four parts, their join included; 4000 tokens, 2/1 heads, window 500: 525 -> 221; 1024 tokens, 4/2 heads, head_dim 128: 210 -> 66.
template <int D>
constexpr int kDkvWavesF32 = D == 64 ? 8 : 4;

template <typename T, int D, bool PARTS>
__global__ __launch_bounds__(64 * kDkvWavesF32<D>) void window_dkv_f32_kernel(WindowParams P) {
  constexpr int NR = 16 * (D / 32), W = kDkvWavesF32<D>;
  __shared__ Sums<2 * NR, W> sums;
  __shared__ f32x4 own[2][D / 8][64];  // the keys' operands, the same in every wavefront
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  WindowParams one = P;  // tiles of 32 keys: one row a token
  one.G = 1;
  const unsigned parts = PARTS ? P.near_parts : 1, part = blockIdx.x / (unsigned)P.Hkv % parts;
  const RowTile t = locate_tile<32, false>(one, blockIdx.x / (unsigned)P.Hkv / parts);
  if (t.s < 0) return;
  const int g = (int)(blockIdx.x % (unsigned)P.Hkv);
  const int u0 = t.tile * 32, u = min(u0 + l32, t.n - 1), last = min(u0 + 31, t.n - 1);
  const int64_t at = ((int64_t)(t.row0 + u) * P.Hkv + g) * D;
  const T* const any = (const T*)P.k + at;
  RowOperand<D> x;
  if (wave < 2) {
    load_row<D>(x, wave == 0 ? any : (const T*)P.v + at, any, hf);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) own[wave][i][lane] = x.x[i];
  }
  __syncthreads();
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) dk[dt] = dv[dt] = zero16();
  const int behind = u0 < P.sinks || t.n - last <= P.window ? t.n : last + P.window;  // the first token that sees none of them
  const int end = behind * P.G;
  auto row = [&](int m) { const int tok = (int)((unsigned)m / (unsigned)P.G); return (int64_t)(t.row0 + tok) * P.Hq + g * P.G + m - tok * P.G; };
  for (int m0 = u0 * P.G + 32 * (int)(part * W + wave); m0 < end; m0 += 32 * (int)(parts * W)) {
    const int m = min(m0 + l32, end - 1);
    const int64_t mine = row(m);
    load_row<D>(x, (const T*)P.q + mine * D, any, hf);
    asm volatile("" ::: "memory");  // the keys' operands are read again each time: kept in registers they would spill others
    const f32x16 sc = dot_rows<D>(x, own[0], lane);
    load_row<D>(x, (const T*)P.d_o + mine * D, any, hf);
    const f32x16 dp = dot_rows<D>(x, own[1], lane);
    // statistics of row m0 + lane%32, passed on to the lanes that hold the row
    const float lse2 = P.lse2[mine], dr = P.dr[mine];
    const int pos = m0 + l32 < end ? (int)((unsigned)m / (unsigned)P.G) : -1;
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
    add_rows<D, T>(dv, p, any, l32, hf, [&](int r) { return m0 + r < end ? (const T*)P.d_o + row(m0 + r) * D : nullptr; });
    add_rows<D, T>(dk, ds, any, l32, hf, [&](int r) { return m0 + r < end ? (const T*)P.q + row(m0 + r) * D : nullptr; });
  }
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      sums.put(wave, 16 * dt + v, lane, dk[dt][v]);
      sums.put(wave, NR + 16 * dt + v, lane, dv[dt][v]);
    }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < W - 1; ++w)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        dk[dt][v] += sums.x[w][16 * dt + v][lane];
        dv[dt][v] += sums.x[w][NR + 16 * dt + v][lane];
      }
  if (PARTS) {
    float* const to = P.parts + (int64_t)blockIdx.x * (2 * NR * 64) + lane;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        to[64 * (16 * dt + v)] = dk[dt][v];
        to[64 * (NR + 16 * dt + v)] = dv[dt][v];
      }
    return;
  }
  if (u0 + l32 < t.n) {
    store_column<D>((T*)P.dk + at, dk, P.scale, hf);
    store_column<D>((T*)P.dv + at, dv, 1.0f, hf);
  }
}
// 32 columns of dK or dV of an item a workgroup, four registers of the parts' sums a thread
template <int D>
__global__ __launch_bounds__(256) void window_dkv_f32_join_kernel(WindowParams P) {
  constexpr int NR = 16 * (D / 32);
  const int vg = threadIdx.x >> 6, lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int dt = blockIdx.y % (D / 32), value = blockIdx.y / (D / 32);
  WindowParams one = P;
  one.G = 1;
  const unsigned tile = blockIdx.x / (unsigned)P.Hkv, g = blockIdx.x % (unsigned)P.Hkv;
  const RowTile t = locate_tile<32, false>(one, tile);
  const int u = t.tile * 32 + l32;
  if (t.s < 0 || u >= t.n) return;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < P.near_parts; ++j) {
    const float* const from = P.parts + ((int64_t)(tile * P.near_parts + j) * P.Hkv + g) * (2 * NR * 64) + 64 * (value * NR + 16 * dt + 4 * vg) + lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += from[64 * e];
  }
  const float f = value ? 1.0f : P.scale;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= f;
  store4((float*)(value ? P.dv : P.dk) + ((int64_t)(t.row0 + u) * P.Hkv + g) * D + 32 * dt + 8 * vg + 4 * hf, x);
}

// ---------------------------------------------------------------------------------------------
// bfloat16 forward.  A workgroup of four wavefronts owns 128 flattened rows of a KV head, 32 a wavefront, and walks the 64-key tiles that any of them sees; K and V tiles are
// shared in LDS and double-buffered by asynchronous loads.  A wavefront takes a tile as two halves of 32 keys, a step of the running softmax each.  A tile that a wavefront's rows
// all see carries no mask; one that none of them sees is only waited for.  256 registers, so two wavefronts share a SIMD, and a CU holds two workgroups (three or four at
// head_dim 64).  What bounds it: at head_dim 128 matrix instructions take 52 to 54 % of the cycles and vector instructions 49 %, about all of them between them, so the one
// wavefront's exponentials hardly run beside the other's matrix instructions; of a wavefront's time 23 % are waits for loads and barriers, 33 % waits for its turn.  The chip keeps
// 1.5 GHz in the longest launches, as under the library's product, whose matrix cores are 75 % busy.  At head_dim 64 it is vector work: 83 % of the cycles, 11.7 instructions per
// matrix instruction.  One sequence of 100001 tokens, 32/8 heads, window 2000: 3.55 ms, 0.92 PFLOP/s; dense causal, 32768 tokens: 8.2 ms, 1.07; 65536 tokens, 14/2 heads, head_dim 64,
// window 1024: 0.31 ms, 0.75.  Measured against it: the halves' products and probabilities interleaved in one wavefront, S1 beside the probabilities of half 0 and O0 beside those
// of half 1: the same at head_dim 128, 0.29 -> 0.36 ms at 64; priorities between the wavefronts: the same; eight wavefronts and 256 rows a workgroup: the same on long sequences, 2039
// tokens in short ones 26 -> 20 us with four.
template <int D, bool PAGED>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void window_fwd_kernel(WindowParams P) {
  __shared__ __attribute__((aligned(1024))) char tiles[2][2][64 * D * 2];  // [buffer][K, V]
  const int splits = PAGED ? P.splits : 1, z = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (unsigned)P.Hkv % (unsigned)splits));
  const RowTile t = locate_tile<32 * kWaves, PAGED>(P, blockIdx.x / (unsigned)P.Hkv / (unsigned)splits);
  if (t.s < 0) return;
  const int g = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % (unsigned)P.Hkv));
  const int64_t from = (int64_t)z * P.per_split, to = z < splits - 1 ? from + P.per_split : 0x7fffffff;
  window_fwd_rows<D, PAGED, kWaves, LoadedTiles<D, PAGED>>(P, &tiles[0][0][0], P, t, g, threadIdx.x & 63, from, to, splits > 1,
                                                           [&](int i, int h, int) __attribute__((always_inline)) { return ((int64_t)z * P.T + t.row0 + i) * P.Hq + h; });
}

// ---------------------------------------------------------------------------------------------
// bfloat16 dQ.  Rows, tiles and their walk as in the forward kernel; a half tile is S, dP and dQ += dS K, whose operands go through one set of registers.  Every row belongs to one
// workgroup here, so this is also where Dr is computed, from the dO in registers and one read of O, and left with LSE for the next kernel.  32768 tokens, 32/8 heads, window 4096: 1.87 ms,
// 1.08 PFLOP/s, matrix cores 63 % busy, vector instructions 42 % of the cycles; 65536 tokens, 14/2 heads, head_dim 64, window 1024: 0.42 ms, 0.84 PFLOP/s, 52 and 67 % (with eight
// wavefronts a workgroup, whose four SIMDs all wait at the same barrier, 0.38 -> 0.48 on another card).
template <int D>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void window_dq_kernel(WindowParams P) {
  constexpr int ROWS = 32 * kWaves, ROW_B = D * 2, TILE_B = 64 * ROW_B, NOP = D / 16;
  __shared__ __attribute__((aligned(1024))) char tiles[2][2][TILE_B];  // [buffer][K, V]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const RowTile t = locate_tile<ROWS, false>(P, blockIdx.x / P.Hkv);
  if (t.s < 0) return;
  const int g = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % (unsigned)P.Hkv));
  const int rows = t.n * P.G, mb = t.tile * ROWS, mw = mb + 32 * wave;
  auto token = [&](int m) { return (int)((unsigned)min(m, rows - 1) / (unsigned)P.G); };
  const int i = token(mw + l32), h = g * P.G + min(mw + l32, rows - 1) - i * P.G;
  auto position = [&](int m) { return __builtin_amdgcn_readfirstlane(token(m)); };  // (see the forward kernel)
  const int ta = position(mb), tb = position(mb + ROWS - 1), wa = position(mw), wb = position(mw + 31);
  const bool working = mw < rows;
  const KeyTiles<64> keys(ta, tb, P.window, P.sinks);
  const int count = keys.count();
  KeySource<D, false> src;
  src.init(P, t, g, max(0, ta - P.window + 1), tb + 1);
  RowsLoader<D, kWaves> loader;
  loader.init(src.pitch, wave, lane);
  const unsigned tiles0 = lds_offset(&tiles[0][0][0]);
  auto issue = [&](int x) __attribute__((always_inline)) {
    int there;
    const unsigned long long o = src.rows_at(P, 64 * keys.at(x) + 64 / kWaves * wave, 64 / kWaves, there);
    const unsigned slot = tiles0 + (x & 1) * 2 * TILE_B;
    loader.issue(src.k + o, there, slot);
    loader.issue(src.v + o, there, slot + TILE_B);
  };
  // B operands of S^T = K Q^T and dP^T = V dO^T: column = row lane%32, slots = d 16ks + 8hf + (0..7)
  bf16x8 qf[NOP], dof[NOP];
  const int64_t row = (int64_t)(t.row0 + i) * P.Hq + h;
  float lse, dr = 0.f;
  {
    const bf16* const qp = (const bf16*)P.q + row * D + 8 * hf;
    const bf16* const dp = (const bf16*)P.d_o + row * D + 8 * hf;
    const bf16* const op = (const bf16*)P.o_in + row * D + 8 * hf;
    bf16x8 of[NOP];
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) { dof[ks] = *(const bf16x8*)(dp + 16 * ks); of[ks] = *(const bf16x8*)(op + 16 * ks); qf[ks] = *(const bf16x8*)(qp + 16 * ks); }
    lse = P.lse[(int64_t)h * P.T + t.row0 + i];
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) dr = __builtin_fmaf((float)dof[ks][e], (float)of[ks][e], dr);
    dr += __shfl_xor(dr, 32, 64);
  }
#pragma unroll
  for (int ks = 0; ks < NOP; ++ks) asm volatile("" : "+v"(qf[ks]), "+v"(dof[ks]));
  asm volatile("" : "+v"(lse), "+v"(dr));
  const float lse2 = lse * 1.4426950408889634f;
  issue(0);

  unsigned row_a[NOP], tr_a[D / 32][2];
#pragma unroll
  for (int ks = 0; ks < NOP; ++ks) row_a[ks] = tiles0 + l32 * ROW_B + 16 * ((2 * ks + hf) ^ chunk_swizzle<D>(l32));
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = 8 * half + 4 * hf + ((lane & 15) >> 2), d = 32 * dt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      tr_a[dt][half] = tiles0 + r * ROW_B + 16 * ((d >> 3) ^ chunk_swizzle<D>(r)) + 2 * (d & 7);
    }
  auto ld_row = [&](int ks, unsigned off) __attribute__((always_inline)) {
    return *(const bf16x8 __attribute__((address_space(3)))*)(uintptr_t)(row_a[ks] + off);
  };
  auto ld_tr = [&](int kk, int dt, unsigned off) __attribute__((always_inline)) {
    const unsigned o = off + kk * 16 * ROW_B;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(tr_a[dt][0] + o));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(tr_a[dt][1] + o));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  bf16x8 op[NOP];
  // Rows with few keys: there O is no average, |O| = |V|, and what its rounding to bf16 moves Dr by is what dS is off by.  Where two tiles hold all keys Dr is taken from them,
  // sum_u P dP in float32 (2039 tokens in short sequences: dQ and dK 0.26 -> 0.24 % off in the 2-norm).
  if (count <= 2) {
    float d = 0.f;
    auto add = [&](auto buf_c) __attribute__((always_inline)) {
      constexpr unsigned BO = decltype(buf_c)::value * 2 * TILE_B;
      const int u0 = 64 * keys.at(decltype(buf_c)::value);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        f32x16 sacc = zero16(), dp = zero16();
#pragma unroll
        for (int ks = 0; ks < NOP; ++ks) sacc = mfma32(ld_row(ks, BO + mt * 32 * ROW_B), qf[ks], sacc);
#pragma unroll
        for (int ks = 0; ks < NOP; ++ks) dp = mfma32(ld_row(ks, BO + TILE_B + mt * 32 * ROW_B), dof[ks], dp);
        const Sight sees(i, u0 + 32 * mt, hf, P.window, P.sinks);
#pragma unroll
        for (int v = 0; v < 16; ++v) d += sees(c_row(v, 0)) ? fast_exp2(__builtin_fmaf(sacc[v], P.scale_log2e, -lse2)) * dp[v] : 0.f;
      }
    };
    if (count == 2) issue(1);
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    add(std::integral_constant<int, 0>());
    if (count == 2) add(std::integral_constant<int, 1>());  // (and is loaded once more below, after a barrier)
    dr = d + __shfl_xor(d, 32, 64);
  }
  if (mw + l32 < rows) P.stats[2 * row + hf] = split3(hf ? dr : lse / P.scale);
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  auto tile = [&](auto buf_c, int u0, bool all) __attribute__((always_inline)) {
    constexpr unsigned BO = decltype(buf_c)::value * 2 * TILE_B;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int ks = 0; ks < NOP; ++ks) op[ks] = ld_row(ks, BO + mt * 32 * ROW_B);  // K rows
      __builtin_amdgcn_sched_barrier(0);
      f32x16 sacc = zero16(), dp = zero16();
#pragma unroll
      for (int ks = 0; ks < NOP; ++ks) {
        sacc = mfma32(op[ks], qf[ks], sacc);
        op[ks] = ld_row(ks, BO + TILE_B + mt * 32 * ROW_B);  // V rows
      }
#pragma unroll
      for (int x = 0; x < NOP; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < NOP; ++ks) {
        dp = mfma32(op[ks], dof[ks], dp);
        op[ks] = ld_tr(2 * mt + ks / (D / 32), ks % (D / 32), BO);  // K^T
      }
      float p[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) p[v] = fast_exp2(__builtin_fmaf(sacc[v], P.scale_log2e, -lse2));
      if (!all) {
        const Sight sees(i, u0 + 32 * mt, hf, P.window, P.sinks);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if (!sees(c_row(v, 0))) { p[v] = 0.f; dp[v] = 0.f; }
        }
      }
      bf16x8 ds[2];
#pragma unroll
      for (int v = 0; v < 16; ++v) ds[v >> 3][v & 7] = (bf16)(p[v] * (dp[v] - dr));
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) acc[dt] = mfma32(op[kk * (D / 32) + dt], ds[kk], acc[dt]);
    }
  };
  auto visit = [&](auto buf_c, int x) __attribute__((always_inline)) {
    const int u0 = 64 * keys.at(x);
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();  // tile x has landed for everyone; everyone is done with tile x - 1
    if (x + 1 < count) issue(x + 1);
    const bool none = !working || u0 > wb || (wa - (u0 + 63) >= P.window && u0 >= P.sinks);
    if (!none) tile(buf_c, u0, u0 + 63 <= wa && (wb - u0 < P.window || u0 + 63 < P.sinks));
  };
  int x = 0;
  for (; x + 2 <= count; x += 2) {
    visit(std::integral_constant<int, 0>(), x);
    visit(std::integral_constant<int, 1>(), x + 1);
  }
  if (x < count) visit(std::integral_constant<int, 0>(), x);
  wait_vmcnt<0>();
  __syncthreads();  // the tiles' LDS is free
  store_tile<D>(&tiles[0][0][0] + wave * 32 * ROW_B, lane, [&](int dt, int v) __attribute__((always_inline)) { return acc[dt][v] * P.scale; },
                [&](int r) __attribute__((always_inline)) -> bf16* {
                  if (mw + r >= rows) return nullptr;
                  const int j = token(mw + r);
                  return (bf16*)P.dq + ((int64_t)(t.row0 + j) * P.Hq + g * P.G + mw + r - j * P.G) * D;
                });
}

// ---------------------------------------------------------------------------------------------
// bfloat16 dK and dV.  A workgroup owns PAIRS * 32 keys of a KV head and walks the flattened rows that see any of them, 32 a stage.  32 keys are the work of two wavefronts on one
// SIMD: the first computes S and P and adds P^T dO to dV, the second, a stage behind, dP and dS = P (dP - Dr) and adds dS^T Q to dK; P goes from one to the other through LDS
// in float32, lane by lane (both hold keys in columns).  Each so needs 150 registers where one wavefront for both would need more than the 256 that let two share a SIMD,
// and has as many matrix instructions as the other.  The second one has the loads to issue besides, and goes first (32768 tokens, 32/8 heads, window 4096: 3.28 -> 2.75 ms; the first
// going first 3.07; the first with the loads 3.17).  What it measures in all, on a card whose library product
// is 5 % slower than on that one: 2.9 ms and 0.93 PFLOP/s there, matrix cores 60 % busy; 65536 tokens, 14/2 heads, head_dim 64: 0.65 ms, 0.72, 50 %.  What took it
// there from 5.15 ms: no spilled registers in the loop (a reload waits for all loads in flight: 7 - 11 ms with a pipeline of two stages that needed 16 more), no integer division in it, LSE
// and Dr subtracted by a step of the matrix product instead of 32 registers and LDS reads of them, and far rows in many short items.
// The stages' Q and dO rows, LSE and Dr come by asynchronous loads, three stages ahead (kFar: two, so that two of its workgroups share a CU's LDS).
//
// Sinks are seen by all rows of their sequence.  The rows behind a sink tile's ordinary ones (far rows) are the work of other workgroups (kFar), far_rows tokens each, that leave their
// sums in float32; the tile's own workgroup, launched after them, adds them in order.  So the result does not depend on who is ahead, and no workgroup has more than its share.
constexpr int kDkvKeys = 128;   // keys of a workgroup, but of kFar
// With more sinks than this their own workgroups take all rows, since there are then sink tiles enough to fill the chip, if KV heads are several.  Backward of 65536 tokens, 32/8 heads, window 1024, with
// far items and without: 4 sinks 4.5 and 10.9 ms, 256: 5.6 and 9.8, 512: 7.0 and 10.2, 1024: 9.8 and 10.6, 2048: 15.1 and 12.1.  (With few heads far items are ahead throughout: 32768 tokens, 8/2
// heads, head_dim 64, 2048 sinks: 0.85 and 2.67 ms.)
constexpr int kFarSinks = 512;
// Far items of a sequence of n tokens: far_blocks blocks of sinks, far_segments each (some may be empty: the first rows of a block's last ones).
// The rows are read once a block, so a block is 64 sinks where there are more than 32 (65536 tokens, 14/2 heads, 64 sinks: 66 us, in two blocks 105).
__host__ __device__ inline int far_keys(int sinks) { return sinks > 32 ? 64 : 32; }
__host__ __device__ inline int far_blocks(int n, int sinks) { return ((sinks < n ? sinks : n) + far_keys(sinks) - 1) / far_keys(sinks); }
__host__ __device__ inline int far_segments(int n, int window, int far_rows) { return far_rows > 0 && n > window ? (n - window + far_rows - 1) / far_rows : 0; }
__host__ __device__ inline int64_t far_items(int n, int window, int sinks, int far_rows) {
  return sinks > kFarSinks ? 0 : (int64_t)far_blocks(n, sinks) * far_segments(n, window, far_rows);
}
// the first token that sees none of the 128 keys around u, but for sinks
__host__ __device__ inline int near_end(int u, int n, int window) {
  const int last = (u | (kDkvKeys - 1)) < n ? (u | (kDkvKeys - 1)) : n - 1;
  return n - last > window ? last + window : n;
}

// Where there are fewer items than the chip works on at a time, an item's rows are shared by near_parts workgroups (kPart) that leave their sums too, which a last launch adds in order
// (kJoin).  2039 tokens in short sequences, 16/2 heads: 186 us whole, 38 and 8 in six parts.
enum DkvMode { kWhole, kFar, kPart, kJoin };
template <int D, int PAIRS, DkvMode MODE>
__global__ __launch_bounds__(128 * PAIRS) __attribute__((amdgpu_waves_per_eu(2))) void window_dkv_kernel(WindowParams P) {
  constexpr int ROW_B = D * 2, TILE_B = 32 * ROW_B, NOP = D / 16, KEYS = 32 * PAIRS, NW = 2 * PAIRS;
  constexpr int kSlots = MODE == kFar ? 4 : 5, kAhead = kSlots - 2, STAT_B = 1024, STAGE_B = 2 * TILE_B;
  constexpr int kNr = 16 * (D / 32);  // accumulator registers
  __shared__ __attribute__((aligned(1024))) char stage[kSlots][STAGE_B];  // Q, dO
  __shared__ __attribute__((aligned(1024))) float pbuf[2][PAIRS][16 * 64];
  __shared__ __attribute__((aligned(1024))) bf16x8 stat[kSlots][64];      // LSE / scale of 32 rows, Dr (split3)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int pair = wave % PAIRS;
  const bool second = wave >= PAIRS;  // wavefronts w and w + 4 share a SIMD
  const int g = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % (unsigned)P.Hkv));
  // which sequence, and what of it
  int s = -1, seq0 = 0, n = 0;
  const unsigned tile_part = blockIdx.x / (unsigned)P.Hkv;
  int64_t x = MODE == kPart ? tile_part / (unsigned)P.near_parts : tile_part, far0 = 0;  // far0: far items of the earlier sequences
  const int64_t tile_id = x;
  for (int base = 0; base < P.S && s < 0; base += 64) {
    int first = 0, len = 0;
    if (base + lane < P.S) { first = P.cu[base + lane]; len = P.cu[base + lane + 1] - first; }
    const int64_t c_far = far_items(len, P.window, P.sinks, P.far_rows);
    const int64_t c = MODE == kFar ? c_far : (int64_t)((len + KEYS - 1) / KEYS);
    int64_t incl = c, incl_far = c_far;
    for (int off = 1; off < 64 && off < P.S - base; off <<= 1) {
      const int64_t a = __shfl_up(incl, off, 64), b = __shfl_up(incl_far, off, 64);
      if (lane >= off) { incl += a; incl_far += b; }
    }
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(base + lane < P.S && x < incl);
    const int src = hit ? __builtin_ctzll(hit) : min(P.S - base, 64) - 1;
    if (hit) {
      s = base + src;
      seq0 = __builtin_amdgcn_readlane(first, src);
      n = __builtin_amdgcn_readlane(len, src);
      x -= __shfl(incl - c, src, 64);
      far0 += __shfl(incl_far - c_far, src, 64);
    } else {
      x -= __shfl(incl, src, 64);
      far0 += __shfl(incl_far, src, 64);
    }
  }
  if (s < 0) return;
  const int segments = far_segments(n, P.window, P.far_rows);
  const int item = __builtin_amdgcn_readfirstlane((int)x);
  int u0, r0, r1;  // first key; rows: tokens r0 .. r1 - 1
  if (MODE == kFar) {
    u0 = item / segments * KEYS;  // (KEYS is far_keys(sinks))
    const int64_t from = (int64_t)near_end(u0, n, P.window) + (int64_t)(item % segments) * P.far_rows;
    if (from >= n) return;
    r0 = (int)from;
    r1 = (int)min(from + P.far_rows, (int64_t)n);
  } else {
    u0 = item * KEYS;
    r0 = u0;
    r1 = (P.sinks > kFarSinks || P.far_rows == 0) && u0 < P.sinks ? n : near_end(u0, n, P.window);
  }
  const int ku = u0 + 32 * pair, kl = min(ku + 31, n - 1);  // this pair's keys (none: ku >= n)
  const int key = min(ku + l32, n - 1);
  // sums left in float32: of a far item [item][KV head][pair][dV, dK][register][lane], of a part [tile][part][KV head][pair][dV, dK][register][lane]
  const int block = far_keys(P.sinks) / 32;  // pairs of a far item
  auto far_sums = [&](int64_t it) { return P.partials + (((it * P.Hkv + g) * block + ku / 32 % block) * 2 + (second ? 1 : 0)) * (kNr * 64) + lane; };
  auto part_sums = [&](int z) { return P.parts + ((((tile_id * P.near_parts + z) * P.Hkv + g) * PAIRS + pair) * 2 + (second ? 1 : 0)) * (kNr * 64) + lane; };
  const bool has_far = MODE != kFar && P.far_rows > 0 && P.sinks <= kFarSinks && ku < min(P.sinks, n);
  const int far_end = near_end(u0, n, P.window), far_count = has_far ? (n - far_end + P.far_rows - 1) / P.far_rows : 0;
  const int64_t far_first = far0 + (int64_t)(ku / far_keys(P.sinks)) * segments;
  if constexpr (MODE == kJoin) {  // 32 columns a workgroup
    const int dt = blockIdx.y;
    float sum[16] = {};
    auto take = [&](const float* from) __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sum[v] += from[(16 * dt + v) * 64];
    };
#pragma unroll 4
    for (int z = 0; z < P.near_parts; ++z) take(part_sums(z));
    for (int z = 0; z < far_count; ++z) take(far_sums(far_first + z));
    if (ku + l32 >= n) return;
    const float f = second ? P.scale : 1.0f;
    bf16* const to = (bf16*)(second ? P.dk : P.dv) + ((int64_t)(seq0 + ku + l32) * P.Hkv + g) * D + 32 * dt + 4 * hf;
#pragma unroll
    for (int vg = 0; vg < 4; ++vg) store4(to + 8 * vg, f32x4{sum[4 * vg] * f, sum[4 * vg + 1] * f, sum[4 * vg + 2] * f, sum[4 * vg + 3] * f});
    return;
  }
  int m0 = r0 * P.G, m1 = r1 * P.G;
  if (MODE == kPart) {
    // tokens in equal shares, of whole stages
    const int z = (int)(tile_part % (unsigned)P.near_parts), share = ((r1 - r0 + P.near_parts - 1) / P.near_parts + 31) / 32 * 32;
    r0 = min(r0 + z * share, r1);
    r1 = min(r0 + share, r1);
    m0 = r0 * P.G;
    m1 = r1 * P.G;
  }
  const int stages = (m1 - m0 + 31) / 32;
  // The stages are walked in a circle from y0 on: where a row's number is a multiple of an ordinary item's rows.  Neighbouring items, which an XCD works on at the same time and which have
  // most of their rows in common, so ask for the same rows at about the same time and meet them in the XCD's L2, which could not hold the rows of one item for the next.
  int y0 = 0;
  if (MODE == kWhole) {
    const int64_t around = ((int64_t)P.window + kDkvKeys) * P.G;
    const int64_t start = (around - m0 % around) % around / 32;
    if (start < stages) y0 = (int)start;
  }

  // The rows of a stage: its first row's token and head, its last row's token.  Carried along, 32 flattened rows at a time: step_t tokens and step_h heads.
  struct Rows {
    int first, head, last;
  };
  const unsigned G = (unsigned)P.G;
  const float inv_g = 1.0f / (float)P.G;
  const int step_t = 32 / (int)G, step_h = 32 % (int)G, last_t = 31 / (int)G, last_h = 31 % (int)G;
  auto rows_from = [&](int y) {
    const int t = __builtin_amdgcn_readfirstlane((int)((unsigned)(32 * y) / G)), h = 32 * y - t * (int)G;
    return Rows{r0 + t, h, r0 + t + last_t + (h + last_h >= P.G ? 1 : 0)};
  };
  auto next_rows = [&](Rows& x) __attribute__((always_inline)) {
    x.first += step_t;
    x.head += step_h;
    if (x.head >= P.G) { x.head -= P.G; ++x.first; }
    x.last = x.first + last_t + (x.head + last_h >= P.G ? 1 : 0);
  };
  // x / G for x < G + 32 (exact: 1 / 2 is further from a multiple of G than the product is off)
  auto token_of = [&](int x) __attribute__((always_inline)) { return (int)(((float)x + 0.5f) * inv_g); };

  // Loads: 32 rows of Q and of dO a stage, RPI rows an instruction; the second wavefronts share them, and the first of these takes the rows' statistics.  A scalar address for the stage's first
  // token, a lane's own row from there on.
  constexpr int C = D / 8, RPI = 64 / C, LOADS = 2 * (32 / RPI), LPW = LOADS / PAIRS;  // load id: tensor id % 2, rows RPI (id / 2) .. of the stage
  static_assert(LPW * PAIRS == LOADS && LPW % 2 == 0, "every second wavefront has as many");
  const unsigned stage0 = lds_offset(&stage[0][0]), stat0 = lds_offset(&stat[0][0]);
  const int wrap = P.Hq - P.G;  // rows of Q from the group's last head of a token to its first of the next, but for one
  int load_y = y0;
  Rows load_rows = rows_from(y0);
  auto issue = [&](int slot) __attribute__((always_inline)) {  // the next stage; in place of rows past the item's last, which are masked, the stage's first
    const int left = m1 - m0 - 32 * load_y;
    const unsigned long long row = (unsigned long long)(seq0 + load_rows.first) * (unsigned)P.Hq + (unsigned)(g * P.G);
    auto row_of = [&](int r) __attribute__((always_inline)) {  // from `row` on
      const int x = load_rows.head + (r < left ? r : 0);
      return (unsigned)x + (unsigned)token_of(x) * (unsigned)wrap;
    };
    unsigned voff = 0;
#pragma unroll
    for (int a = 0; a < LPW; ++a) {
      const int id = pair * LPW + a, r = id / 2 * RPI + lane / C;
      if (a % 2 == 0) voff = row_of(r) * (D * 2) + 16 * ((lane % C) ^ chunk_swizzle<D>(r));  // (the next one is the other tensor's)
      const unsigned long long base = (unsigned long long)(id % 2 ? P.d_o : P.q) + row * (D * 2);
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" : : "v"(voff), "s"(stage0 + slot * STAGE_B + id % 2 * TILE_B + id / 2 * 1024), "s"(base) : "memory", "m0");
    }
    if (pair == 0) {
      const unsigned off = row_of(l32) * 32 + hf * 16;
      const unsigned long long base = (unsigned long long)P.stats + row * 32;
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" : : "v"(off), "s"(stat0 + slot * STAT_B), "s"(base) : "memory", "m0");
    }
    next_rows(load_rows);
    if (++load_y == stages) {
      load_y = 0;
      load_rows = rows_from(0);
    }
  };

  // B operand: K or V rows; column = key lane%32, slots = d 16ks + 8hf + (0..7)
  bf16x8 kv[NOP];
  {
    const bf16* kp = (const bf16*)(second ? P.v : P.k) + ((int64_t)(seq0 + key) * P.Hkv + g) * D + 8 * hf;
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) kv[ks] = *(const bf16x8*)(kp + 16 * ks);
  }
#pragma unroll
  for (int ks = 0; ks < NOP; ++ks) asm volatile("" : "+v"(kv[ks]));
  if (second) {
#pragma unroll
    for (int x = 0; x < kAhead; ++x)
      if (x < stages) issue(x);
  }

  // Rows of Q (dO for the second wavefront), transposed reads of the other.  The chunk of a row that an operand needs differs from that of the first one in bits that the
  // swizzle leaves to be turned over, so one address serves all.
  const unsigned row_a = stage0 + (second ? TILE_B : 0) + l32 * ROW_B + 16 * (hf ^ chunk_swizzle<D>(l32));
  const unsigned tr_a = stage0 + (second ? 0 : TILE_B) + [&] {
    const int r = 4 * hf + ((lane & 15) >> 2), d = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    return r * ROW_B + 16 * ((d >> 3) ^ chunk_swizzle<D>(r)) + 2 * (d & 7);
  }();
  auto ld_row = [&](int ks, unsigned off) __attribute__((always_inline)) {
    return *(const bf16x8 __attribute__((address_space(3)))*)(uintptr_t)((row_a + off) ^ (32 * ks));
  };
  auto ld_tr = [&](int kk, int dt, unsigned off) __attribute__((always_inline)) {
    const unsigned at = (tr_a + off) ^ (64 * dt);
    static_assert(D == 128 || D == 64, "rows 8 further: the swizzle turns chunk bit 1");
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(at + kk * 16 * ROW_B));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4 __attribute__((address_space(3)))*)(uintptr_t)((at ^ 32) + (kk * 16 + 8) * ROW_B));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const unsigned stat_a = stat0 + (second ? 512 : 0) + l32 * 16;
  auto ld_stat = [&](int slot) __attribute__((always_inline)) { return *(const bf16x8 __attribute__((address_space(3)))*)(uintptr_t)(stat_a + slot * STAT_B); };
  bf16x8 minus = zero_bf16x8();  // B operand that subtracts what split3 made
  if (hf == 0) minus[0] = minus[1] = minus[2] = (bf16)-1.0f;
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();

  // before stage x of the loop: stages x and x + 1 are there, and what the next loads replace is no longer read
  int load_slot = kAhead;
  auto turn = [&](int x) __attribute__((always_inline)) {
    if (second) {
      if (x + kAhead > stages) wait_vmcnt<0>();
      else if (pair == 0) wait_vmcnt<(kAhead - 2) * (LPW + 1)>();  // the stages behind x + 1 may still be on their way
      else wait_vmcnt<(kAhead - 2) * LPW>();
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the probabilities are written, the operands read
    __builtin_amdgcn_s_barrier();
    if (second && x + kAhead < stages) {
      issue(load_slot);
      load_slot = load_slot == kSlots - 1 ? 0 : load_slot + 1;
    }
  };
  // One set of operand registers goes through both contractions: every register is refilled with an operand of the next one when its matrix instruction has been issued, so that LDS is
  // read at an even pace and no product waits for operands; the steps are fenced.
  bf16x8 op[NOP], less;
  auto add = [&](const bf16x8 (&w)[2], int next) __attribute__((always_inline)) {  // acc += transposed x w; then rows of slot `next`
#pragma unroll
    for (int x = 0; x < NOP; ++x) {
      acc[x % (D / 32)] = mfma32(op[x], w[x / (D / 32)], acc[x % (D / 32)]);
      op[x] = ld_row(x, next * STAGE_B);
      if (x == 0) less = ld_stat(next);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto product = [&](int slot) __attribute__((always_inline)) {  // S - LSE / scale, or dP - Dr (the subtraction is one more step of the contraction); then transposed operands
    f32x16 c = mfma32(less, minus, zero16());
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) {
      c = mfma32(op[ks], kv[ks], c);
      op[ks] = ld_tr(ks / (D / 32), ks % (D / 32), slot * STAGE_B);
      __builtin_amdgcn_sched_barrier(0);
    }
    return c;
  };
  auto after = [](int slot) { return slot == kSlots - 1 ? 0 : slot + 1; };
  int slot = 0;
  turn(0);
  if (!second) {
    // stage x: S(x); P(x); dV += P(x)^T dO(x)
    less = ld_stat(0);
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) op[ks] = ld_row(ks, 0);
    int y = y0;
    Rows at_rows = rows_from(y0);
    for (int x = 0; x < stages; ++x) {
      const f32x16 s = product(slot);
      float p[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) p[v] = fast_exp2(s[v] * P.scale_log2e);
      const int left = m1 - m0 - 32 * y;  // rows that exist
      const bool all = at_rows.first >= kl && (at_rows.last - ku < P.window || kl < P.sinks) && left >= 32;
      if (!all) {
        // Row r of the stage is (head + r) / G tokens behind the first, so it sees the key if lo <= r < hi without any division: (key - first) G <= head + r < (key - first + window) G
        const int64_t behind = key - at_rows.first, until = key < P.sinks ? 64 : behind + P.window;
        auto bound = [&](int64_t tokens) { return (int)max(min(tokens, (int64_t)64), (int64_t)-1) * P.G - at_rows.head - 4 * hf; };
        int lo = bound(behind), hi = min(bound(until), left - 4 * hf);
        asm volatile("" : "+v"(lo), "+v"(hi));  // (else the compiler keeps row numbers in registers around the loop)
#pragma unroll
        for (int v = 0; v < 16; ++v) p[v] = (c_row(v, 0) >= lo) & (c_row(v, 0) < hi) ? p[v] : 0.f;
      }
      bf16x8 w[2];
#pragma unroll
      for (int v = 0; v < 16; ++v) w[v >> 3][v & 7] = (bf16)p[v];
#pragma unroll
      for (int vg = 0; vg < 4; ++vg) *(f32x4*)&pbuf[x & 1][pair][(vg * 64 + lane) * 4] = f32x4{p[4 * vg], p[4 * vg + 1], p[4 * vg + 2], p[4 * vg + 3]};
      __builtin_amdgcn_sched_barrier(0);
      slot = after(slot);
      add(w, slot);
      next_rows(at_rows);
      if (++y == stages) {
        y = 0;
        at_rows = rows_from(0);
      }
      turn(x + 1);
    }
  } else {
    // stage x: dK += dS(x - 2)^T Q(x - 2); dP(x - 1); dS(x - 1).  So its matrix instructions come while the other wavefront has its exponentials.
    __builtin_amdgcn_s_setprio(2);
    bf16x8 w[2] = {zero_bf16x8(), zero_bf16x8()};
#pragma unroll
    for (int ks = 0; ks < NOP; ++ks) op[ks] = zero_bf16x8();
    for (int x = 1; x <= stages; ++x) {
      turn(x);
      add(w, slot);
      const f32x16 dp = product(slot);
#pragma unroll
      for (int vg = 0; vg < 4; ++vg) {
        const f32x4 p = *(const f32x4*)&pbuf[(x - 1) & 1][pair][(vg * 64 + lane) * 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[vg >> 1][4 * (vg & 1) + e] = (bf16)(p[e] * dp[4 * vg + e]);
      }
      slot = after(slot);
    }
    add(w, 0);
  }
  wait_vmcnt<0>();

  if (MODE == kFar || MODE == kPart) {
    float* const to = MODE == kFar ? far_sums(far0 + item) : part_sums((int)(tile_part % (unsigned)P.near_parts));
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) to[(16 * dt + v) * 64] = acc[dt][v];
    return;
  }
  for (int z = 0; z < far_count; ++z) {
    const float* const from = far_sums(far_first + z);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[dt][v] += from[(16 * dt + v) * 64];
  }
  __syncthreads();  // the stages' LDS is free
  static_assert(NW * 32 * ROW_B <= (int)sizeof(stage), "every wavefront's rows");
  char* const buf = &stage[0][0] + wave * 32 * ROW_B;
  const float f = second ? P.scale : 1.0f;
  store_tile<D>(buf, lane, [&](int dt, int v) __attribute__((always_inline)) { return acc[dt][v] * f; },
                [&](int r) __attribute__((always_inline)) -> bf16* {
                  return ku + r < n ? (bf16*)(second ? P.dk : P.dv) + ((int64_t)(seq0 + ku + r) * P.Hkv + g) * D : nullptr;
                });
}

// ---------------------------------------------------------------------------------------------
int check_rows(int64_t tokens, int G) {
  if (tokens * G > 0x7fffffffll - 512) { set_error("%lld tokens of %d query heads per KV head pass 32 bits", (long long)tokens, G); return SB_ERR_UNSUPPORTED; }
  return SB_OK;
}
int64_t row_tiles(const int32_t* cu, int S, int G, int rows) {
  int64_t n = 0;
  for (int s = 0; s < S; ++s) n += ((int64_t)(cu[s + 1] - cu[s]) * G + rows - 1) / rows;
  return n;
}
int64_t row_tiles_most(int total, int S, int G, int rows) { return ((int64_t)total * G) / rows + S; }

int grid_of(int64_t workgroups, int threads, dim3* grid) {
  if (workgroups * threads > 0xffffffffll) { set_error("too many tiles for one launch"); return SB_ERR_UNSUPPORTED; }
  *grid = dim3((unsigned)workgroups);
  return SB_OK;
}
int check_aligned(const void* const* p, int n) {
  for (int i = 0; i < n; ++i)
    if ((uintptr_t)p[i] % 16 != 0) { set_error("a buffer does not start at a multiple of 16 bytes"); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}

int launch_window_fwd(const WindowParams& P, int D, int dtype, bool paged, int64_t tiles, hipStream_t st) {
  const int64_t items = tiles * P.Hkv * (paged ? P.splits : 1);
  dim3 grid;
  const int rc = grid_of(items, dtype == SB_F32 ? 256 : 64 * kWaves, &grid);
  if (rc != SB_OK) return rc;
  auto launch = [&](auto d, auto pg) {
    constexpr int DD = decltype(d)::value;
    constexpr bool PAGED = decltype(pg)::value;
    if (dtype == SB_F32) hipLaunchKernelGGL((window_fwd_f32_kernel<float, DD, PAGED>), grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL((window_fwd_kernel<DD, PAGED>), grid, dim3(64 * kWaves), 0, st, P);
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
  return check_rows(g->T, g->G);
}
static WindowParams window_params(const Geo& g, const sb_problem* p, int32_t window, int32_t sinks) {
  WindowParams P{};
  P.cu = p->cu_seqlens_dev;
  P.T = g.T; P.S = g.S; P.Hq = g.Hq; P.Hkv = g.Hkv; P.G = g.G;
  P.window = window; P.sinks = sinks;
  P.scale = g.softmax_scale; P.scale_log2e = g.softmax_scale * 1.4426950408889634f;
  return P;
}

static int64_t longest(const int32_t* cu, int S) {
  int64_t n = 0;
  for (int s = 0; s < S; ++s)
    if (cu[s + 1] - cu[s] > n) n = cu[s + 1] - cu[s];
  return n;
}
// Far rows a far item takes: short enough that a long sequence's sinks are many workgroups' work, and no more than 64 of them to a block of sinks, whose sums its own workgroup adds.  None
// where all of a sequence is at most twice an ordinary item's rows: a launch of their own costs more than the sinks' workgroups are longer then.  Backward of one sequence, 16/2 heads, 4 sinks,
// without far items and with them: window 512, 2 times its rows 74 and 121 us, 3 times 99 and 127, 4 times 150 and 141; window 2048, 1.5 times 262 and 258 us, 2 times 440 and 332, 3 times 905 and 458.
// (Batches of many sequences with 32/8 heads fill the chip either way: with them 0 to 6 % less time from 1.2 to 3 times, 16 % at 4.)
static int far_rows_of(int64_t longest, int window) {
  if (longest <= 2 * ((int64_t)window + kDkvKeys)) return 0;
  const int64_t rows = (longest - window + 63) / 64;
  return rows < 256 ? 256 : (int)((rows + 31) / 32 * 32);
}
struct WindowWs { size_t lse2, dr, stats, partials, parts, bytes; int64_t far; int far_rows, near_parts; };
static WindowWs window_bwd_ws(const Geo& g, const int32_t* cu, int window, int sinks) {
  WindowWs w{};
  size_t o = 0;
  const size_t rows = (size_t)g.T * g.Hq, f32 = g.dtype == SB_F32 ? 1 : 0;
  w.lse2 = o;  o = align_up(o + sizeof(float) * rows * f32);
  w.dr = o;    o = align_up(o + sizeof(float) * rows * f32);
  w.stats = o; o = align_up(o + 2 * sizeof(bf16x8) * rows * (1 - f32));
  const int64_t n = longest(cu, g.S);
  w.far_rows = far_rows_of(n, window);
  if (g.dtype == SB_BF16)
    for (int s = 0; s < g.S; ++s) w.far += far_items(cu[s + 1] - cu[s], window, sinks, w.far_rows);
  w.partials = o; o = align_up(o + (size_t)w.far * g.Hkv * 2 * far_keys(sinks) * g.D * sizeof(float));
  // Parts where items are fewer than workgroups fit the chip (a CU's LDS holds one at head_dim 128, two at 64): up to 8, of 16 stages at least
  w.near_parts = 1;
  if (g.dtype == SB_BF16) {
    const int64_t items = row_tiles(cu, g.S, 1, kDkvKeys) * g.Hkv;
    const int64_t most = n < (int64_t)window + kDkvKeys ? n : (int64_t)window + kDkvKeys;  // tokens of an item
    int64_t parts = items > 0 ? (g.D == 128 ? 256 : 512) / items : 1;
    if (parts > most * g.G / (32 * 16)) parts = most * g.G / (32 * 16);
    if (parts > 8) parts = 8;
    if (parts > 1) w.near_parts = (int)parts;
    w.parts = o;
    if (parts > 1) o = align_up(o + (size_t)items * parts * 2 * kDkvKeys * g.D * sizeof(float));
  } else {
    // float32: the same from four strips of 32 rows a wavefront on.  (The sinks' keys are seen by all rows.)
    const int64_t items = row_tiles(cu, g.S, 1, 32) * g.Hkv, waves = g.D == 64 ? kDkvWavesF32<64> : kDkvWavesF32<128>;
    const int64_t most = sinks > 0 || n < (int64_t)window + 32 ? n : (int64_t)window + 32, strips = most * g.G / 32;
    int64_t parts = items > 0 && strips >= 4 * waves ? 256 / items : 1;
    if (parts > strips / waves) parts = strips / waves;
    if (parts > 8) parts = 8;
    if (parts > 1) w.near_parts = (int)parts;
    w.parts = o;
    if (parts > 1) o = align_up(o + (size_t)items * parts * 2 * 32 * g.D * sizeof(float));
  }
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
  if (bwd_bytes) *bwd_bytes = (int64_t)window_bwd_ws(g, p->cu_seqlens_host, window, sinks).bytes;
  return SB_OK;
}

int sb_window_attn_fwd(const sb_problem* p, int32_t window, int32_t sinks, const void* q, const void* k, const void* v, void* o, float* lse, void* ws,
                       void* stream) {
  Geo g;
  int rc = check_window(p, window, sinks, &g);
  if (rc != SB_OK) return rc;
  if (g.T == 0) return SB_OK;
  if (!p->cu_seqlens_dev) { set_error("cu_seqlens_dev is required"); return SB_ERR_INVALID_ARG; }
  if (!q || !k || !v || !o || !lse) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  const void* const buffers[] = {q, k, v, o};
  if ((rc = check_aligned(buffers, 4)) != SB_OK) return rc;
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
  const void* const buffers[] = {q, k, v, o, d_o, dq, dk, dv, ws};
  if ((rc = check_aligned(buffers, 9)) != SB_OK) return rc;
  const hipStream_t st = (hipStream_t)stream;
  WindowParams P = window_params(g, p, window, sinks);
  P.q = q; P.k = k; P.v = v; P.o_in = o; P.lse = (float*)lse; P.d_o = d_o; P.dq = dq; P.dk = dk; P.dv = dv;
  const int32_t* cu = p->cu_seqlens_host;
  const WindowWs w = window_bwd_ws(g, cu, window, sinks);
  P.lse2 = (float*)((char*)ws + w.lse2);
  P.dr = (float*)((char*)ws + w.dr);
  P.stats = (bf16x8*)((char*)ws + w.stats);
  P.partials = (float*)((char*)ws + w.partials);
  P.far_rows = w.far_rows;
  P.parts = (float*)((char*)ws + w.parts);
  P.near_parts = w.near_parts;
  const bool f32 = g.dtype == SB_F32;
  const int64_t rows = (int64_t)g.T * g.Hq, per = 1024 / g.D;
  const int64_t q_items = row_tiles(cu, g.S, g.G, forward_rows(g.dtype)) * g.Hkv, k_items = row_tiles(cu, g.S, 1, f32 ? 32 : kDkvKeys) * g.Hkv;
  dim3 delta_grid, q_grid, k_grid, far_grid, part_grid;
  if ((f32 && (rc = grid_of((rows + per - 1) / per, 256, &delta_grid)) != SB_OK) || (rc = grid_of(q_items, 256, &q_grid)) != SB_OK ||
      (rc = grid_of(k_items, 4 * kDkvKeys, &k_grid)) != SB_OK || (rc = grid_of(w.far * g.Hkv, 4 * far_keys(sinks), &far_grid)) != SB_OK ||
      (rc = grid_of(k_items * w.near_parts, 4 * kDkvKeys, &part_grid)) != SB_OK)
    return rc;
  auto launch = [&](auto d) {
    constexpr int D = decltype(d)::value;
    {
      KernelTimer kt(K_WINDOW_DQ, st);
      if (f32) {
        hipLaunchKernelGGL((window_delta_kernel<float, D>), delta_grid, dim3(256), 0, st, P, rows);
        SB_LAUNCH_CHECK("window_delta_kernel");
        hipLaunchKernelGGL((window_dq_f32_kernel<float, D>), q_grid, dim3(256), 0, st, P);
      } else {
        hipLaunchKernelGGL((window_dq_kernel<D>), q_grid, dim3(64 * kWaves), 0, st, P);
      }
      SB_LAUNCH_CHECK("window_dq_kernel");
    }
    KernelTimer kt(K_WINDOW_DKV, st);
    if (f32) {
      constexpr int threads = 64 * kDkvWavesF32<D>;
      if (w.near_parts > 1) {
        hipLaunchKernelGGL((window_dkv_f32_kernel<float, D, true>), part_grid, dim3(threads), 0, st, P);
        SB_LAUNCH_CHECK("window_dkv_f32_kernel");
        hipLaunchKernelGGL((window_dkv_f32_join_kernel<D>), dim3(k_grid.x, 2 * (D / 32)), dim3(256), 0, st, P);
      } else {
        hipLaunchKernelGGL((window_dkv_f32_kernel<float, D, false>), k_grid, dim3(threads), 0, st, P);
      }
    } else {
      if (w.far > 0) {
        if (far_keys(sinks) == 32) hipLaunchKernelGGL((window_dkv_kernel<D, 1, kFar>), far_grid, dim3(128), 0, st, P);
        else hipLaunchKernelGGL((window_dkv_kernel<D, 2, kFar>), far_grid, dim3(256), 0, st, P);
        SB_LAUNCH_CHECK("window_dkv_kernel, far rows");
      }
      if (w.near_parts > 1) {
        hipLaunchKernelGGL((window_dkv_kernel<D, kDkvKeys / 32, kPart>), part_grid, dim3(kDkvKeys * 4), 0, st, P);
        SB_LAUNCH_CHECK("window_dkv_kernel, parts");
        hipLaunchKernelGGL((window_dkv_kernel<D, kDkvKeys / 32, kJoin>), dim3(k_grid.x, D / 32), dim3(kDkvKeys * 4), 0, st, P);
      } else {
        hipLaunchKernelGGL((window_dkv_kernel<D, kDkvKeys / 32, kWhole>), k_grid, dim3(kDkvKeys * 4), 0, st, P);
      }
    }
    SB_LAUNCH_CHECK("window_dkv_kernel");
    return (int)SB_OK;
  };
  return g.D == 128 ? launch(std::integral_constant<int, 128>()) : launch(std::integral_constant<int, 64>());
}

}  // extern "C"
