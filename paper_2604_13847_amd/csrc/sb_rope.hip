// Rotary positions of packed batches (one position a token, or one of every axis), and the append of new tokens to a paged cache, which is the same kernel with another destination.
//
// Pair (x, y) of a head becomes A (x cos a - y sin a, y cos a + x sin a), a = 2 pi pos turns_i.  The product is taken in float64 and reduced to
// half a revolution either way before it is rounded, so an angle is off by 2^-24 of that at any position; products and sums are in
// float32, rounded once to the tensors' type.
//
// Memory-bound: every element is read and written once.  A wavefront takes a token at a time: each lane works out one pair's angle (a float64
// product and one sine and cosine), which all heads of the token then share through LDS, and handles units of 2 VEC elements, VEC pairs,
// of one head after the other, with kBatch heads' loads in flight.  65536 tokens, 32/8 heads, head_dim 128, bfloat16: 282 us, 4.8 TB/s, where a copy of
// 2 GiB reaches 4.95 (stores past the caches: 426 us).  The append of 64 single tokens takes 6 us, of 8192 new tokens 36 us (5.6 TB/s: most of it stays in the
// last-level cache).
#include <math.h>

#include <type_traits>

#include "sb_rope.h"

namespace sb {

struct RopeParams {
  const void *q, *k, *v;
  void *q_out, *k_out;                    // k_out: unless paged
  int64_t q_pitch, k_pitch, v_pitch;      // elements from token to token
  const int32_t *positions, *cu;          // positions: null: index in the sequence, `cached` added
  int T, S, Hq, Hkv, heads;               // heads: units of work of a token: Hq (0 without q) + Hkv (0 without k) + Hkv (v)
  int rot;
  float amplitude, sign;
  PagedCache cache;                       // paged only
  const int32_t* cached;
  int max_new;
  int run;                                // tokens a wavefront takes
  const int32_t* axis_positions;          // [axes][T]: with AXES
  uint8_t axis[SB_ROPE_MAX_PAIRS];
  double turns[SB_ROPE_MAX_PAIRS];
};

template <typename T, int N> struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Vec { T x[N]; };

// PAGED: k and v go to the cache's pages.  VEC 8: rot is a multiple of 16 and everything is 16-byte aligned, so a unit is two 16-byte pieces
// (float: 32 bytes); else single pairs.  AXES: every pair's position is that of its axis; each lane loads its own.
template <typename T, int D, int VEC, bool HALF, bool PAGED, bool AXES>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams P) {
  constexpr int UNITS = D / 2 / VEC;          // of a head
  constexpr int PER = 64 / (UNITS < 64 ? UNITS : 64);  // heads a wavefront handles at a time
  constexpr int kBatch = VEC == 8 ? 4 : 2;
  using V = Vec<T, VEC>;
  __shared__ __attribute__((aligned(16))) float2 table[4][SB_ROPE_MAX_PAIRS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int u = lane % UNITS, first_head = lane / UNITS;
  const bool turned = VEC * u < P.rot / 2;
  // elements of the unit's two pieces; (what is not turned is copied in two pieces too)
  const int rest = P.rot + 2 * (VEC * u - P.rot / 2);
  const int at_a = HALF ? (turned ? VEC * u : rest) : 2 * VEC * u, at_b = HALF && turned ? at_a + P.rot / 2 : at_a + VEC;
  const int64_t tok0 = ((int64_t)blockIdx.x * 4 + wave) * P.run;
  float2* const cs = table[wave];
  const double turns = lane < P.rot / 2 ? P.turns[lane] : 0.0;
  const int32_t* const axis_positions = AXES ? P.axis_positions + (lane < P.rot / 2 ? (int64_t)P.axis[lane] * P.T : 0) : nullptr;
  int s = 0, first = 0, behind = -1;  // the token's sequence, its first row and the one behind its last
  for (int64_t tok = tok0; tok < min(tok0 + P.run, (int64_t)P.T); ++tok) {
    int64_t pos = 0;
    if (PAGED || (!AXES && !P.positions)) {
      if (tok >= behind) {
        s = sequence_of(P.cu, P.S, (int)tok, lane);
        if (s >= P.S) break;  // behind the last sequence
        first = P.cu[s];
        behind = P.cu[s + 1];
      }
      pos = tok - first;
      if (PAGED) {
        if (pos < 0 || pos >= P.max_new) continue;
        pos += max(P.cached[s], 0);
      }
    } else if (!AXES) {
      pos = P.positions[tok];
    }
    {
      double t = (double)(AXES ? axis_positions[tok] : pos) * turns;
      t -= rint(t);
      float sn, cn;
      sincospif(2.0f * (float)t, &sn, &cn);
      cs[lane] = make_float2(cn * P.amplitude, sn * P.amplitude * P.sign);
    }
    asm volatile("" ::: "memory");  // (LDS operations of a wavefront complete in order)
    float cn[VEC], sn[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float2 x = cs[(VEC * u + e) & (SB_ROPE_MAX_PAIRS - 1)];
      cn[e] = x.x; sn[e] = x.y;
    }
    asm volatile("" ::: "memory");
    T *page_k = nullptr, *page_v = nullptr;
    if (PAGED) {
      const int64_t row = P.cache.row_of(s, pos, 0);
      if (row >= 0) { page_k = (T*)P.cache.k + row * D; page_v = (T*)P.cache.v + row * D; }
    }
    const int hq = P.q ? P.Hq : 0, hk = hq + (P.k ? P.Hkv : 0);
    for (int h0 = first_head; h0 < P.heads; h0 += PER * kBatch) {
      V a[kBatch], b[kBatch];
      T* to[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int h = h0 + i * PER;
        to[i] = nullptr;
        if (h < P.heads) {
          const T* from;
          if (h < hq) {
            from = (const T*)P.q + tok * P.q_pitch + h * D;
            to[i] = (T*)P.q_out + (tok * P.Hq + h) * D;
          } else if (h < hk) {
            const int g = h - hq;
            from = (const T*)P.k + tok * P.k_pitch + g * D;
            to[i] = PAGED ? (page_k ? page_k + (int64_t)g * P.cache.page_size * D : nullptr) : (T*)P.k_out + (tok * P.Hkv + g) * D;
          } else {
            const int g = h - hk;
            from = (const T*)P.v + tok * P.v_pitch + g * D;
            to[i] = page_v ? page_v + (int64_t)g * P.cache.page_size * D : nullptr;
          }
          a[i] = *(const V*)(from + at_a);
          b[i] = *(const V*)(from + at_b);
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (!to[i]) continue;
        if (turned && h0 + i * PER < hk) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            // pair e of the unit: (a[e], b[e]), or elements 2e, 2e + 1 of the two pieces in a row
            T& xr = HALF ? a[i].x[e] : 2 * e < VEC ? a[i].x[(2 * e) % VEC] : b[i].x[(2 * e) % VEC];
            T& yr = HALF ? b[i].x[e] : 2 * e + 1 < VEC ? a[i].x[(2 * e + 1) % VEC] : b[i].x[(2 * e + 1) % VEC];
            const float x = (float)xr, y = (float)yr;
            // (written out, so that every form of the kernel rounds alike)
            xr = (T)__builtin_fmaf(x, cn[e], -(y * sn[e]));
            yr = (T)__builtin_fmaf(y, cn[e], x * sn[e]);
          }
        }
        *(V*)(to[i] + at_a) = a[i];
        *(V*)(to[i] + at_b) = b[i];
      }
    }
  }
}

int check_rope(const sb_rope* r, int head_dim) {
  if (r->rot_dim < 2 || r->rot_dim % 2 != 0 || r->rot_dim > head_dim) {
    set_error("rot_dim %d must be even and in 2 .. head_dim (%d)", r->rot_dim, head_dim);
    return SB_ERR_INVALID_ARG;
  }
  if (r->layout != SB_ROPE_HALF && r->layout != SB_ROPE_INTERLEAVED) { set_error("bad rope layout %d", r->layout); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}

int check_axes(const sb_rope* r, const sb_rope_axes* a, const int32_t* positions) {
  if (!r || !a || !positions) { set_error("a rope, its axes and their positions are required"); return SB_ERR_INVALID_ARG; }
  if (a->num_axes < 1 || a->num_axes > SB_ROPE_MAX_AXES) { set_error("num_axes %d must be in 1 .. %d", a->num_axes, SB_ROPE_MAX_AXES); return SB_ERR_INVALID_ARG; }
  for (int i = 0; i < r->rot_dim / 2; ++i)
    if (a->axis[i] >= a->num_axes) { set_error("pair %d is of axis %d: there are %d", i, a->axis[i], a->num_axes); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}

int check_pitch(const char* what, int64_t* pitch, int64_t contiguous) {
  if (*pitch == 0) *pitch = contiguous;
  if (*pitch < contiguous) { set_error("%s_pitch %lld is less than a token's %lld elements", what, (long long)*pitch, (long long)contiguous); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}

template <typename T, int D, int VEC, bool PAGED>
static void launch_layout(const RopeParams& P, bool half, dim3 grid, hipStream_t st) {
  auto launch = [&](auto h, auto axes) {
    hipLaunchKernelGGL((rope_kernel<T, D, VEC, decltype(h)::value, PAGED, decltype(axes)::value>), grid, dim3(256), 0, st, P);
  };
  auto with_axes = [&](auto h) { if (P.axis_positions) launch(h, std::true_type()); else launch(h, std::false_type()); };
  if (half) with_axes(std::true_type()); else with_axes(std::false_type());
}
template <typename T, bool PAGED>
static void launch_rope(const RopeParams& P, int D, bool half, bool wide, dim3 grid, hipStream_t st) {
  if (D == 128) {
    if (wide) launch_layout<T, 128, 8, PAGED>(P, half, grid, st); else launch_layout<T, 128, 1, PAGED>(P, half, grid, st);
  } else {
    if (wide) launch_layout<T, 64, 8, PAGED>(P, half, grid, st); else launch_layout<T, 64, 1, PAGED>(P, half, grid, st);
  }
}

static int enqueue_rope(RopeParams& P, int D, int dtype, bool half, bool paged, hipStream_t st) {
  const int esize = dtype == SB_F32 ? 4 : 2;
  const bool wide = P.rot % 16 == 0 && aligned16(P.q) && aligned16(P.k) && aligned16(P.v) && aligned16(P.q_out) && aligned16(P.k_out) &&
                    aligned16(P.cache.k) && aligned16(P.cache.v) && P.q_pitch * esize % 16 == 0 && P.k_pitch * esize % 16 == 0 &&
                    P.v_pitch * esize % 16 == 0;
  P.run = P.T / 8192 < 1 ? 1 : P.T / 8192 > 8 ? 8 : P.T / 8192;
  if (P.T >> 25 > P.run) P.run = P.T >> 25;  // (a launch has fewer than 2^32 threads)
  const dim3 grid((unsigned)(((int64_t)P.T + 4 * P.run - 1) / (4 * P.run)));
  KernelTimer kt(K_ROPE, st);
  if (dtype == SB_F32) {
    if (paged) launch_rope<float, true>(P, D, half, wide, grid, st); else launch_rope<float, false>(P, D, half, wide, grid, st);
  } else {
    if (paged) launch_rope<bf16, true>(P, D, half, wide, grid, st); else launch_rope<bf16, false>(P, D, half, wide, grid, st);
  }
  SB_LAUNCH_CHECK("rope_kernel");
  return SB_OK;
}

static void set_rope(RopeParams* P, const sb_rope* r) {
  P->rot = r->rot_dim;
  P->amplitude = r->amplitude;
  for (int i = 0; i < r->rot_dim / 2; ++i) P->turns[i] = r->turns[i];
}
static void set_axes(RopeParams* P, const sb_rope* r, const sb_rope_axes* a, const int32_t* positions) {
  P->axis_positions = positions;
  for (int i = 0; i < r->rot_dim / 2; ++i) P->axis[i] = a->axis[i];
}

}  // namespace sb

using namespace sb;

extern "C" {

int sb_rope_init(sb_rope* out, int32_t rot_dim, int32_t layout, double base, int32_t scaling, double factor, double original_length, double low,
                 double high) {
  if (!out) { set_error("null rope"); return SB_ERR_INVALID_ARG; }
  sb_rope r{};
  r.rot_dim = rot_dim; r.layout = layout; r.amplitude = 1.0f;
  const int rc = check_rope(&r, 2 * SB_ROPE_MAX_PAIRS);
  if (rc != SB_OK) return rc;
  if (scaling < SB_ROPE_PLAIN || scaling > SB_ROPE_BANDS) { set_error("bad rope scaling %d", scaling); return SB_ERR_INVALID_ARG; }
  if (!(base > 1.0) || !isfinite(base)) { set_error("base must be a number above 1"); return SB_ERR_INVALID_ARG; }
  if (scaling != SB_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) { set_error("factor must be at least 1"); return SB_ERR_INVALID_ARG; }
  const bool parts = scaling == SB_ROPE_YARN || scaling == SB_ROPE_BANDS;
  if (parts) {
    if (!(low > 0.0)) low = 1.0;
    if (!(high > 0.0)) high = scaling == SB_ROPE_YARN ? 32.0 : 4.0;
    if (!(original_length > 0.0) || !isfinite(original_length)) { set_error("original_length must be a positive number"); return SB_ERR_INVALID_ARG; }
    if (!(low < high) || !isfinite(high)) { set_error("low (%g) must be less than high (%g)", low, high); return SB_ERR_INVALID_ARG; }
  }
  if (scaling == SB_ROPE_NTK) {
    if (rot_dim < 4) { set_error("SB_ROPE_NTK needs a rot_dim of at least 4"); return SB_ERR_INVALID_ARG; }
    base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  }
  const double two_pi = 6.283185307179586476925;
  double from = 0.0, width = 1.0;  // SB_ROPE_YARN: the pairs between the two bounds
  if (scaling == SB_ROPE_YARN) {
    // pair that turns x times in original_length tokens
    auto pair = [&](double x) { return rot_dim * log(original_length / (x * two_pi)) / (2.0 * log(base)); };
    const double lo = fmax(floor(pair(high)), 0.0), hi = fmin(ceil(pair(low)), (double)(rot_dim - 1));
    from = lo;
    width = fmax(hi - lo, 1e-3);
    r.amplitude = (float)(0.1 * log(factor) + 1.0);
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rot_dim);
    double slow = 0.0;  // share that is divided by the factor
    if (scaling == SB_ROPE_LINEAR) slow = 1.0;
    if (scaling == SB_ROPE_YARN) slow = fmin(fmax((i - from) / width, 0.0), 1.0);
    if (scaling == SB_ROPE_BANDS) slow = 1.0 - fmin(fmax((original_length * f / two_pi - low) / (high - low), 0.0), 1.0);
    if (slow > 0.0) f = f / factor * slow + f * (1.0 - slow);
    r.turns[i] = f / two_pi;
  }
  *out = r;
  return SB_OK;
}

static int rope_apply(const sb_problem* p, const sb_rope* r, const sb_rope_axes* axes, bool with_axes, const int32_t* positions, const void* q, int64_t q_pitch, const void* k,
                      int64_t k_pitch, void* q_out, void* k_out, int direction, void* stream) {
  Geo g;
  int rc = make_batch(p, &g);
  if (rc != SB_OK) return rc;
  if (!r) { set_error("null rope"); return SB_ERR_INVALID_ARG; }
  if ((rc = check_rope(r, g.D)) != SB_OK || (with_axes && (rc = check_axes(r, axes, positions)) != SB_OK)) return rc;
  if (direction != SB_ROPE_FORWARD && direction != SB_ROPE_BACKWARD) { set_error("bad direction %d", direction); return SB_ERR_INVALID_ARG; }
  if ((rc = check_pitch("q", &q_pitch, (int64_t)g.Hq * g.D)) != SB_OK || (rc = check_pitch("k", &k_pitch, (int64_t)g.Hkv * g.D)) != SB_OK) return rc;
  if (!q != !q_out || !k != !k_out) { set_error("an input without its output, or the other way round"); return SB_ERR_INVALID_ARG; }
  if ((q && q == q_out && q_pitch != (int64_t)g.Hq * g.D) || (k && k == k_out && k_pitch != (int64_t)g.Hkv * g.D)) {
    set_error("in place needs contiguous tokens");
    return SB_ERR_INVALID_ARG;
  }
  if (g.T == 0 || (!q && !k)) return SB_OK;
  if (!positions && !p->cu_seqlens_dev) { set_error("cu_seqlens_dev is required without positions"); return SB_ERR_INVALID_ARG; }
  RopeParams P{};
  P.q = q; P.k = k; P.q_out = q_out; P.k_out = k_out; P.q_pitch = q_pitch; P.k_pitch = k_pitch;
  P.positions = positions; P.cu = p->cu_seqlens_dev;
  P.T = g.T; P.S = g.S; P.Hq = g.Hq; P.Hkv = g.Hkv; P.heads = (q ? g.Hq : 0) + (k ? g.Hkv : 0);
  P.sign = direction == SB_ROPE_FORWARD ? 1.0f : -1.0f;
  set_rope(&P, r);
  if (with_axes) set_axes(&P, r, axes, positions);
  return enqueue_rope(P, g.D, g.dtype, r->layout == SB_ROPE_HALF, false, (hipStream_t)stream);
}

int sb_rope_apply(const sb_problem* p, const sb_rope* r, const int32_t* positions, const void* q, int64_t q_pitch, const void* k, int64_t k_pitch,
                  void* q_out, void* k_out, int direction, void* stream) {
  return rope_apply(p, r, nullptr, false, positions, q, q_pitch, k, k_pitch, q_out, k_out, direction, stream);
}

int sb_rope_axes_init(sb_rope_axes* out, int32_t num_axes, const int32_t* pairs, int32_t order) {
  if (!out || !pairs) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if (num_axes < 1 || num_axes > SB_ROPE_MAX_AXES) { set_error("num_axes %d must be in 1 .. %d", num_axes, SB_ROPE_MAX_AXES); return SB_ERR_INVALID_ARG; }
  if (order != SB_AXES_SECTIONS && order != SB_AXES_IN_TURN) { set_error("bad order of axes %d", order); return SB_ERR_INVALID_ARG; }
  int left[SB_ROPE_MAX_AXES], total = 0;
  for (int a = 0; a < num_axes; ++a) {
    if (pairs[a] < 0 || pairs[a] > SB_ROPE_MAX_PAIRS - total) { set_error("pairs of axes must be 0 .. %d in all", SB_ROPE_MAX_PAIRS); return SB_ERR_INVALID_ARG; }
    total += left[a] = pairs[a];
  }
  if (total == 0) { set_error("no axis has any pair"); return SB_ERR_INVALID_ARG; }
  sb_rope_axes x{};
  x.num_axes = num_axes;
  for (int i = 0; i < total;)
    for (int a = 0; a < num_axes; ++a)
      for (int n = order == SB_AXES_SECTIONS ? left[a] : left[a] > 0 ? 1 : 0; n > 0; --n, --left[a]) x.axis[i++] = (uint8_t)a;
  for (int i = total; i < SB_ROPE_MAX_PAIRS; ++i) x.axis[i] = (uint8_t)num_axes;  // (so that a rope of more pairs than the axes have is refused)
  *out = x;
  return SB_OK;
}

int sb_rope_join(sb_rope* out, const sb_rope* ropes, int32_t num_ropes) {
  if (!out || !ropes) { set_error("null rope"); return SB_ERR_INVALID_ARG; }
  if (num_ropes < 1) { set_error("at least one rope is needed"); return SB_ERR_INVALID_ARG; }
  sb_rope r = ropes[0];
  r.rot_dim = 0;
  int at = 0;
  for (int a = 0; a < num_ropes; ++a) {
    const int rc = check_rope(&ropes[a], 2 * SB_ROPE_MAX_PAIRS);
    if (rc != SB_OK) return rc;
    if (ropes[a].layout != r.layout || ropes[a].amplitude != r.amplitude) { set_error("joined ropes need one layout and one amplitude"); return SB_ERR_INVALID_ARG; }
    const int n = ropes[a].rot_dim / 2;
    if (n > SB_ROPE_MAX_PAIRS - at) { set_error("joined ropes have more than %d pairs", SB_ROPE_MAX_PAIRS); return SB_ERR_INVALID_ARG; }
    for (int i = 0; i < n; ++i) r.turns[at++] = ropes[a].turns[i];
  }
  for (int i = at; i < SB_ROPE_MAX_PAIRS; ++i) r.turns[i] = 0.0;
  r.rot_dim = 2 * at;
  *out = r;
  return SB_OK;
}

int sb_rope_axes_apply(const sb_problem* p, const sb_rope* r, const sb_rope_axes* axes, const int32_t* positions, const void* q, int64_t q_pitch, const void* k, int64_t k_pitch,
                       void* q_out, void* k_out, int direction, void* stream) {
  return rope_apply(p, r, axes, true, positions, q, q_pitch, k, k_pitch, q_out, k_out, direction, stream);
}

static int cache_append(const sb_cache* c, const sb_chunk* n, const sb_rope* r, const sb_rope_axes* axes, bool with_axes, const int32_t* positions, const void* q, int64_t q_pitch,
                        const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* q_out, void* stream) {
  int rc = check_cache(c, n);
  if (rc != SB_OK) return rc;
  const int D = c->head_dim, Hq = n->num_q_heads, Hkv = c->num_kv_heads;
  if ((r && (rc = check_rope(r, D)) != SB_OK) || (with_axes && (rc = check_axes(r, axes, positions)) != SB_OK)) return rc;
  if ((rc = check_pitch("q", &q_pitch, (int64_t)Hq * D)) != SB_OK || (rc = check_pitch("k", &k_pitch, (int64_t)Hkv * D)) != SB_OK ||
      (rc = check_pitch("v", &v_pitch, (int64_t)Hkv * D)) != SB_OK)
    return rc;
  if (!q != !q_out) { set_error("q without q_out, or the other way round"); return SB_ERR_INVALID_ARG; }
  if (q && q == q_out && q_pitch != (int64_t)Hq * D) { set_error("in place needs contiguous tokens"); return SB_ERR_INVALID_ARG; }
  if (n->total_new == 0 || n->num_seqs == 0) return SB_OK;
  if (!k || !v) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if ((rc = check_cache_arrays(c, n)) != SB_OK) return rc;
  RopeParams P{};
  P.q = q; P.k = k; P.v = v; P.q_out = q_out; P.q_pitch = q_pitch; P.k_pitch = k_pitch; P.v_pitch = v_pitch;
  P.cu = n->cu_new; P.cached = n->cached; P.max_new = n->max_new;
  P.T = n->total_new; P.S = n->num_seqs; P.Hq = Hq; P.Hkv = Hkv; P.heads = (q ? Hq : 0) + 2 * Hkv;
  P.sign = 1.0f;
  P.cache = make_paged(c);
  if (r) set_rope(&P, r);
  if (with_axes) set_axes(&P, r, axes, positions);
  return enqueue_rope(P, D, c->dtype, !r || r->layout == SB_ROPE_HALF, true, (hipStream_t)stream);
}

int sb_cache_append(const sb_cache* c, const sb_chunk* n, const sb_rope* r, const void* q, int64_t q_pitch, const void* k, int64_t k_pitch,
                    const void* v, int64_t v_pitch, void* q_out, void* stream) {
  return cache_append(c, n, r, nullptr, false, nullptr, q, q_pitch, k, k_pitch, v, v_pitch, q_out, stream);
}

int sb_cache_append_axes(const sb_cache* c, const sb_chunk* n, const sb_rope* r, const sb_rope_axes* axes, const int32_t* positions, const void* q, int64_t q_pitch, const void* k,
                         int64_t k_pitch, const void* v, int64_t v_pitch, void* q_out, void* stream) {
  return cache_append(c, n, r, axes, true, positions, q, q_pitch, k, k_pitch, v, v_pitch, q_out, stream);
}

}  // extern "C"
