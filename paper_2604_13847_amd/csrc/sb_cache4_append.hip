// Append of new tokens to a paged cache in four bits: keys turned by their positions, keys and values rounded to four bits, queries turned.
//
// Memory-bound: q is read and written once, k and v are read once and written in a third of their size (and once more where the caller asks for the values as held).  A workgroup takes a
// token at a time, each of its four wavefronts every fourth batch of heads.
//
// What four bits a key gets must not depend on how its turn is computed (in another order of operations an element next to a threshold would get another code), so angles, sines and the
// turn itself are float64, rounded to float32 once.  Sine and cosine come from their Taylor series on an eighth of a revolution either way, eight terms each: off by less than 2^-45.
// The thresholds between codes are a step of six bits times a number of at most three, exact in float32.
#include <math.h>

#include <type_traits>

#include "sb_cache4.h"
#include "sb_rope.h"

namespace sb {

struct Append4Params {
  const void *q, *k, *v;
  void *q_out, *k_held, *v_held;
  int64_t q_pitch, k_pitch, v_pitch;  // elements from token to token
  const int32_t *cu, *cached, *axis_positions;  // axis_positions [axes][T], or null: cached + i
  int T, S, Hq, Hkv, max_new;
  int rot;
  float amplitude;
  PagedCache4 cache;
  int run;  // tokens a workgroup takes
  uint8_t axis[SB_ROPE_MAX_PAIRS];
  double turns[SB_ROPE_MAX_PAIRS];
};

// cos and sin of 2 pi t, |t| <= 1/2
__device__ inline double2 turn_of(double t) {
  const double quarter = rint(4.0 * t);
  const double x = 6.283185307179586476925 * (t - 0.25 * quarter), y = x * x;  // |x| <= pi / 4
  double s = -1.0 / 1307674368000.0, c = -1.0 / 87178291200.0;
  s = __builtin_fma(s, y, 1.0 / 6227020800.0);
  c = __builtin_fma(c, y, 1.0 / 479001600.0);
  s = __builtin_fma(s, y, -1.0 / 39916800.0);
  c = __builtin_fma(c, y, -1.0 / 3628800.0);
  s = __builtin_fma(s, y, 1.0 / 362880.0);
  c = __builtin_fma(c, y, 1.0 / 40320.0);
  s = __builtin_fma(s, y, -1.0 / 5040.0);
  c = __builtin_fma(c, y, -1.0 / 720.0);
  s = __builtin_fma(s, y, 1.0 / 120.0);
  c = __builtin_fma(c, y, 1.0 / 24.0);
  s = __builtin_fma(s, y, -1.0 / 6.0);
  c = __builtin_fma(c, y, -0.5);
  s = __builtin_fma(s * y, x, x);
  c = __builtin_fma(c, y, 1.0);
  const int n = (int)quarter & 3;
  const double cs = n & 1 ? s : c, sn = n & 1 ? c : s;
  return make_double2(n == 1 || n == 2 ? -cs : cs, n >= 2 ? -sn : sn);
}

// 1/6 of the largest magnitude (its bits: numbers that are none are above all others), rounded to six significant bits; the bits of the bfloat16
__device__ inline unsigned step_of(unsigned largest) {
  if (largest >= 0x7f800000u) return 0x7fc00000u;
  const float sixth = __uint_as_float(largest) * 0.16666667163372040f;
  const unsigned r = (__float_as_uint(sixth) + 0x20000u) & ~0x3ffffu;
  return min(r, 0x7e280000u);  // 1.3125 * 2^125
}
// The code of the number nearest x / step, ties to the even code
__device__ inline unsigned code_of(float x, float step) {
  const float y = fabsf(x);
  const unsigned level = (y > 0.25f * step) + (y >= 0.75f * step) + (y > 1.25f * step) + (y >= 1.75f * step) + (y > 2.5f * step) + (y >= 3.5f * step) + (y > 5.0f * step);
  return level | (__float_as_uint(x) >> 31 << 3);
}
__device__ inline float level_of(unsigned code) {
  const unsigned m = code & 7;
  const float y = m < 4 ? 0.5f * (float)m : m < 6 ? (float)m - 2.0f : 2.0f * (float)m - 8.0f;
  return code & 8 ? -y : y;
}

template <typename T> __device__ inline void load8(float (&x)[8], const T* from, bool wide) {
  T y[8];
  if (wide) {
    typedef struct alignas(16) { T x[16 / sizeof(T)]; } Piece;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(Piece*)(y + i * 16 / sizeof(T)) = ((const Piece*)from)[i];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = from[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)y[e];
}
template <typename T> __device__ inline void store8(T* to, const float (&x)[8]) {  // 16-byte aligned
  typedef struct alignas(16) { T x[16 / sizeof(T)]; } Piece;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    Piece p;
#pragma unroll
    for (int e = 0; e < (int)(16 / sizeof(T)); ++e) p.x[e] = (T)x[i * (16 / sizeof(T)) + e];
    ((Piece*)to)[i] = p;
  }
}

// A lane holds eight neighbouring elements, 8 x .. 8 x + 7 of a head (x = lane % (D/8)); four lanes a group of 32.  WIDE: rows of q, k, v are 16-byte aligned.
template <typename T, int D, bool HALF, bool TURN, bool WIDE>
__global__ __launch_bounds__(256) void cache4_append_kernel(Append4Params P) {
  constexpr int LPH = D / 8, PER = 64 / LPH;  // lanes a head, heads a wavefront takes at a time
  __shared__ double2 table[4][SB_ROPE_MAX_PAIRS];
  __shared__ __attribute__((aligned(16))) unsigned codes[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int x = lane % LPH, sub = lane / LPH;
  double2* const cs = table[wave];
  const double turns = TURN && lane < P.rot / 2 ? P.turns[lane] : 0.0;
  const int32_t* const axis_positions = P.axis_positions ? P.axis_positions + (lane < P.rot / 2 ? (int64_t)P.axis[lane] * P.T : 0) : nullptr;
  const int heads = (P.q ? P.Hq : 0) + 2 * P.Hkv, hv = P.Hkv;  // in this order: k, v, q
  const int64_t tok0 = (int64_t)blockIdx.x * P.run;
  int s = 0, first = 0, behind = -1;
  for (int64_t tok = tok0; tok < min(tok0 + P.run, (int64_t)P.T); ++tok) {
    if (tok >= behind) {
      s = sequence_of(P.cu, P.S, (int)tok, lane);
      if (s >= P.S) break;  // behind the last sequence
      first = P.cu[s];
      behind = P.cu[s + 1];
    }
    int64_t pos = tok - first;
    if (pos < 0 || pos >= P.max_new) continue;
    pos += max(P.cached[s], 0);
    if (TURN) {
      double t = (double)(axis_positions ? axis_positions[tok] : pos) * turns;
      t -= rint(t);
      const double2 z = turn_of(t);
      cs[lane] = make_double2(z.x * (double)P.amplitude, z.y * (double)P.amplitude);
    }
    asm volatile("" ::: "memory");  // (LDS operations of a wavefront complete in order)
    const int64_t row0 = P.cache.row_of(s, pos, 0);
    for (int h0 = wave * PER; h0 < heads; h0 += 4 * PER) {
      const int h = h0 + sub;
      const bool there = h < heads;
      const int kind = !there ? 3 : h < hv ? 0 : h < 2 * hv ? 1 : 2, g = kind == 0 ? h : kind == 1 ? h - hv : h - 2 * hv;
      const T* const from = kind == 0 ? (const T*)P.k + tok * P.k_pitch + g * D : kind == 1 ? (const T*)P.v + tok * P.v_pitch + g * D
                            : kind == 2 ? (const T*)P.q + tok * P.q_pitch + g * D : nullptr;
      float a[8] = {};
      if (there) load8(a, from + 8 * x, WIDE);
      if (TURN && (kind == 0 || kind == 2)) {
        // the other elements of the pairs: another eight (HALF), or these themselves
        float b[8];
        if (HALF) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int d = 8 * x + e, half = P.rot / 2;
            b[e] = d < P.rot ? (float)from[d < half ? d + half : d - half] : 0.f;
          }
        }
        float r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = 8 * x + e, half = P.rot / 2;
          const bool is_x = HALF ? d < half : (e & 1) == 0;
          const int pair = HALF ? (d < half ? d : d - half) : d >> 1;
          const double2 z = cs[pair & (SB_ROPE_MAX_PAIRS - 1)];
          const float mine = a[e], other = HALF ? b[e] : a[e ^ 1];
          if (kind == 0) r[e] = (float)((double)mine * z.x + (double)other * (is_x ? -z.y : z.y));
          else r[e] = __builtin_fmaf(mine, (float)z.x, other * (float)(is_x ? -z.y : z.y));
          if (d >= P.rot) r[e] = mine;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = r[e];
      }
      if (kind == 2) store8((T*)P.q_out + (tok * P.Hq + g) * D + 8 * x, a);
      // (all lanes take part in what follows)
      unsigned largest = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(a[e]) & 0x7fffffffu);
      largest = max(largest, (unsigned)__shfl_xor((int)largest, 1, 64));
      largest = max(largest, (unsigned)__shfl_xor((int)largest, 2, 64));
      const unsigned bits = step_of(largest);
      const float step = __uint_as_float(bits);
      unsigned word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) word |= code_of(a[e], step) << 4 * e;
      if (!(step > 0.f)) word = 0;
      codes[wave][lane] = word;
      asm volatile("" ::: "memory");
      if (kind < 2) {
        if (row0 >= 0) {
          const int64_t row = row0 + (int64_t)g * P.cache.page_size;
          if (x % 4 == 0) ((unsigned short*)(kind == 0 ? P.cache.k_step : P.cache.v_step))[row * (D / 32) + x / 4] = (unsigned short)(bits >> 16);
          if (kind == 0) {
            *(unsigned*)(P.cache.k + row * (D / 2) + (x % 4) * (D / 8) + 4 * (x / 4)) = word;
          } else {  // word i of 16, the head's lanes two (D = 64: half) a word
#pragma unroll
            for (int i = x; i < 16; i += LPH) {
              unsigned w = 0;
#pragma unroll
              for (int j = 0; j < D / 16; ++j) w |= (codes[wave][sub * LPH + 2 * j + (i >> 3)] >> 4 * (i & 7) & 15u) << 4 * j;
              if (D == 128) *(unsigned*)(P.cache.v + row * (D / 2) + 4 * i) = w;
              else *(unsigned short*)(P.cache.v + row * (D / 2) + 2 * i) = (unsigned short)w;
            }
          }
        }
        T* const held = (T*)(kind == 0 ? P.k_held : P.v_held);
        if (held) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = level_of(word >> 4 * e & 15u) * step;
          store8(held + (tok * P.Hkv + g) * D + 8 * x, y);
        }
      }
      asm volatile("" ::: "memory");
    }
  }
}

int check_cache4(const sb_cache4* c, const sb_chunk* n) {
  if (!c) { set_error("null cache or chunk"); return SB_ERR_INVALID_ARG; }
  const sb_cache like{c->num_pages, c->page_size, c->num_kv_heads, c->head_dim, c->dtype, c->max_pages, c->k, c->v, c->page_table};
  return check_cache(&like, n);
}
int check_cache4_arrays(const sb_cache4* c, const sb_chunk* n) {
  const sb_cache like{c->num_pages, c->page_size, c->num_kv_heads, c->head_dim, c->dtype, c->max_pages, c->k, c->v, c->page_table};
  if (c->num_pages > 0 && (!c->k_step || !c->v_step)) { set_error("pages without an address"); return SB_ERR_INVALID_ARG; }
  return check_cache_arrays(&like, n);
}
PagedCache4 make_paged(const sb_cache4* c) {
  return PagedCache4{(unsigned char*)c->k, (unsigned char*)c->v, (bf16*)c->k_step, (bf16*)c->v_step, c->page_table, c->num_pages, c->max_pages, c->page_size,
                     __builtin_ctz((unsigned)c->page_size), c->num_kv_heads};
}

}  // namespace sb

using namespace sb;

extern "C" int sb_cache4_append(const sb_cache4* c, const sb_chunk* n, const sb_rope* r, const sb_rope_axes* axes, const int32_t* positions, const void* q, int64_t q_pitch,
                                const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* q_out, void* k_held, void* v_held, void* stream) {
  int rc = check_cache4(c, n);
  if (rc != SB_OK) return rc;
  const int D = c->head_dim, Hq = n->num_q_heads, Hkv = c->num_kv_heads;
  if ((r && (rc = check_rope(r, D)) != SB_OK) || ((axes || positions) && (rc = check_axes(r, axes, positions)) != SB_OK)) return rc;
  if ((rc = check_pitch("q", &q_pitch, (int64_t)Hq * D)) != SB_OK || (rc = check_pitch("k", &k_pitch, (int64_t)Hkv * D)) != SB_OK ||
      (rc = check_pitch("v", &v_pitch, (int64_t)Hkv * D)) != SB_OK)
    return rc;
  if (!q != !q_out) { set_error("q without q_out, or the other way round"); return SB_ERR_INVALID_ARG; }
  if (n->total_new == 0 || n->num_seqs == 0) return SB_OK;
  if (!k || !v) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if ((rc = check_cache4_arrays(c, n)) != SB_OK) return rc;
  // (several lanes read what one of them overwrites)
  if ((q && q == q_out) || k == k_held || v == v_held) { set_error("outputs in the place of inputs are not supported"); return SB_ERR_INVALID_ARG; }
  if (!aligned16(q_out) || !aligned16(k_held) || !aligned16(v_held) || !aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_step) || !aligned16(c->v_step)) {
    set_error("a buffer does not start at a multiple of 16 bytes");
    return SB_ERR_INVALID_ARG;
  }
  Append4Params P{};
  P.q = q; P.k = k; P.v = v; P.q_out = q_out; P.k_held = k_held; P.v_held = v_held; P.q_pitch = q_pitch; P.k_pitch = k_pitch; P.v_pitch = v_pitch;
  P.cu = n->cu_new; P.cached = n->cached; P.max_new = n->max_new; P.axis_positions = positions;
  P.T = n->total_new; P.S = n->num_seqs; P.Hq = Hq; P.Hkv = Hkv;
  P.cache = make_paged(c);
  if (r) {
    P.rot = r->rot_dim;
    P.amplitude = r->amplitude;
    for (int i = 0; i < r->rot_dim / 2; ++i) { P.turns[i] = r->turns[i]; P.axis[i] = axes ? axes->axis[i] : 0; }
  }
  const int esize = c->dtype == SB_F32 ? 4 : 2;
  const bool wide = aligned16(q) && aligned16(k) && aligned16(v) && q_pitch * esize % 16 == 0 && k_pitch * esize % 16 == 0 && v_pitch * esize % 16 == 0;
  P.run = P.T / 2048 < 1 ? 1 : P.T / 2048 > 8 ? 8 : P.T / 2048;
  if (P.T >> 23 > P.run) P.run = P.T >> 23;  // (a launch has fewer than 2^32 threads)
  const dim3 grid((unsigned)(((int64_t)P.T + P.run - 1) / P.run));
  const hipStream_t st = (hipStream_t)stream;
  KernelTimer kt(K_ROPE, st);
  auto launch = [&](auto t, auto d, auto half, auto turn, auto w) {
    hipLaunchKernelGGL((cache4_append_kernel<decltype(t), decltype(d)::value, decltype(half)::value, decltype(turn)::value, decltype(w)::value>), grid, dim3(256), 0, st, P);
  };
  auto with_w = [&](auto t, auto d, auto half, auto turn) { if (wide) launch(t, d, half, turn, std::true_type()); else launch(t, d, half, turn, std::false_type()); };
  auto with_r = [&](auto t, auto d) {
    if (!r) with_w(t, d, std::true_type(), std::false_type());
    else if (r->layout == SB_ROPE_HALF) with_w(t, d, std::true_type(), std::true_type());
    else with_w(t, d, std::false_type(), std::true_type());
  };
  auto with_d = [&](auto t) { if (D == 128) with_r(t, std::integral_constant<int, 128>()); else with_r(t, std::integral_constant<int, 64>()); };
  if (c->dtype == SB_F32) with_d(float()); else with_d(bf16());
  SB_LAUNCH_CHECK("cache4_append_kernel");
  return SB_OK;
}
