// Attention with a sliding window and sinks, forward and backward, over packed batches or (forward) over a paged cache.
//
//   S = scale Q K^T,  row t sees u <= t with t - u < window or u < sinks,  P = softmax(S),  O = P V,  LSE = log sum exp S
//   Dr = rowsum(dO * O),  dP = dO V^T,  dS = P * (dP - Dr),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// All products are computed with the query (forward, dQ) or the key (dK/dV) in a column of the matrix instructions' result, as S^T = K Q^T: statistics are then
// per lane, and a result is the next product's operand without any cross-lane movement (c_row).
#include <math.h>

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

int launch_window_fwd(const WindowParams& P, int D, int dtype, bool paged, int64_t tiles32, int64_t tiles, hipStream_t st) {
  const int64_t items = tiles32 * P.Hkv;
  dim3 grid;
  const int rc = grid_of((items + 3) / 4, &grid);
  if (rc != SB_OK) return rc;
  return with_types(D, dtype, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int DD = decltype(d)::value;
    if (paged) hipLaunchKernelGGL((window_fwd_f32_kernel<T, DD, true>), grid, dim3(256), 0, st, P, items);
    else hipLaunchKernelGGL((window_fwd_f32_kernel<T, DD, false>), grid, dim3(256), 0, st, P, items);
    SB_LAUNCH_CHECK("window_fwd_f32_kernel");
    return SB_OK;
  });
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
  return launch_window_fwd(P, g.D, g.dtype, false, row_tiles(p->cu_seqlens_host, g.S, g.G, 32), 0, (hipStream_t)stream);
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
