// Append of new tokens to a paged cache in four bits: keys turned by their positions, keys and values rounded to four bits, queries turned.
//
// Memory-bound: q is read and written once, k and v are read once and written in a third of their size (and once more where the caller asks for the values as held).  A
// wavefront takes a token at a time (or, of few tokens, every fourth batch of heads of one), the next heads' loads on their way.  8192 tokens, 32/8 heads of 128, values as held too: 53 us, 3.9
// TB/s (a copy of as many bytes: 42); 143 with a wavefront to a batch of heads, which computed the angles again for every one of them.
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
  int waves;  // to a token: 4 or 1
  int run;    // tokens of these, one after the other
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
// The code of the number nearest x / step, ties to the even code: at the thresholds of even levels (0.75, 1.75, 3.5 steps) the upper one, at the others the lower one.  Three comparisons, each
// with a threshold that goes by those before.
__device__ inline unsigned code_of(float x, float step) {
  const float y = fabsf(x), t1 = 0.25f * step, t2 = 0.75f * step, t3 = 1.25f * step, t4 = 1.75f * step, t5 = 2.5f * step, t6 = 3.5f * step, t7 = 5.0f * step;
  const bool c4 = y >= t4;
  const float even = c4 ? t6 : t2, low = c4 ? t5 : t1, high = c4 ? t7 : t3;
  const bool c2 = y >= even;
  const float odd = c2 ? high : low;
  return (unsigned)c4 * 4 + (unsigned)c2 * 2 + (unsigned)(y > odd) + (__float_as_uint(x) >> 31 << 3);
}
// Eight neighbouring elements as they lie in memory
template <typename T> struct alignas(16) Eight { T x[8]; };
template <typename T, bool WIDE> __device__ inline Eight<T> load8(const T* from) {
  if (WIDE) return *(const Eight<T>*)from;
  Eight<T> y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y.x[e] = from[e];
  return y;
}
__device__ inline void store8(bf16* to, const float (&x)[8]) {  // 16-byte aligned
  bf16x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (bf16)x[e];
  *(bf16x8*)to = y;
}
__device__ inline void store8(float* to, const float (&x)[8]) {
  *(f32x4*)to = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(to + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// A lane holds eight neighbouring elements, 8 x .. 8 x + 7 of a head (x = lane % (D/8)); four lanes a group of 32.  WIDE: rows of q, k, v are 16-byte aligned, and (HALF) what a lane's
// elements are paired with is eight neighbours too.
template <typename T, int D, bool HALF, bool TURN, bool WIDE>
__global__ __launch_bounds__(256) void cache4_append_kernel(Append4Params P) {
  constexpr int LPH = D / 8, PER = 64 / LPH;  // lanes a head, heads a wavefront takes at a time
  // What every element of a head is multiplied with, and what its other one is; element 8 x + e at 16 e + x (D/8 e + x), so that lanes side by side read places side by side
  __shared__ double2 table[4][TURN ? D : 1];
  __shared__ float2 table_q[4][TURN ? D : 1];
  __shared__ __attribute__((aligned(16))) unsigned codes[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int x = lane % LPH, sub = lane / LPH, half = P.rot / 2;
  double2* const cs = table[wave];
  float2* const cs_q = table_q[wave];
  const double turns = TURN && lane < half ? P.turns[lane] : 0.0;
  const int32_t* const axis_positions = P.axis_positions ? P.axis_positions + (lane < half ? (int64_t)P.axis[lane] * P.T : 0) : nullptr;
  const int kv_units = (P.Hkv + PER - 1) / PER, units = 2 * kv_units + (P.q ? (P.Hq + PER - 1) / PER : 0);  // of PER heads: k, v, q
  const bool turned = TURN && 8 * x < P.rot;       // some of the lane's elements are
  // the two elements of pair `lane`, and their places in the tables
  auto place = [](int d) { return (d & 7) * LPH + (d >> 3); };
  const int place_a = place(HALF ? lane : 2 * lane), place_b = place(HALF ? lane + half : 2 * lane + 1);
  if (TURN)
    for (int d = P.rot + lane; d < D; d += 64) {  // what is not turned
      cs[place(d)] = make_double2(1.0, 0.0);
      cs_q[place(d)] = make_float2(1.f, 0.f);
    }
  const int away = !HALF ? 0 : 8 * x < half ? half : -half;  // where their others are (WIDE)
  const int step = P.waves, unit0 = step == 1 ? 0 : wave;
  const int64_t tok0 = (step == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x) * P.run;
  int s = 0, first = 0, behind = -1;
  Eight<T> mine{}, other{}, next{}, next_other{};
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
    const int64_t row0 = P.cache.row_of(s, pos, 0);
    double t = TURN ? (double)(axis_positions ? axis_positions[tok] : pos) * turns : 0.0;
    bool ready = !TURN;
    auto kind_of = [&](int u) { return u < kv_units ? 0 : u < 2 * kv_units ? 1 : 2; };  // k, v, q
    auto load = [&](int u, Eight<T>& a, Eight<T>& b) __attribute__((always_inline)) {
      const int kind = kind_of(u), g = (u - kind * kv_units) * PER + sub;
      if (u >= units || g >= (kind == 2 ? P.Hq : P.Hkv)) return;
      const T* const from = (kind == 0 ? (const T*)P.k + tok * P.k_pitch : kind == 1 ? (const T*)P.v + tok * P.v_pitch : (const T*)P.q + tok * P.q_pitch) + g * D + 8 * x;
      a = load8<T, WIDE>(from);
      if (HALF && turned && kind != 1) {
        if (WIDE) {
          b = load8<T, true>(from + away);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int d = 8 * x + e;
            b.x[e] = d < P.rot ? from[d < half ? half + e : e - half] : (T)0.f;
          }
        }
      }
    };
    load(unit0, mine, other);
    for (int u = unit0; u < units; u += step) {
      const int kind = kind_of(u), g = (u - kind * kv_units) * PER + sub;
      const bool there = g < (kind == 2 ? P.Hq : P.Hkv);
      load(u + step, next, next_other);
      if (!ready) {  // (while the loads are on their way)
        t -= rint(t);
        double2 z = turn_of(t);
        z.x *= (double)P.amplitude;
        z.y *= (double)P.amplitude;
        if (lane < half) {
          cs[place_a] = make_double2(z.x, -z.y);
          cs[place_b] = z;
          cs_q[place_a] = make_float2((float)z.x, -(float)z.y);
          cs_q[place_b] = make_float2((float)z.x, (float)z.y);
        }
        ready = true;
      }
      asm volatile("" ::: "memory");  // (LDS operations of a wavefront complete in order)
      float a[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = there ? (float)mine.x[e] : 0.f;
      if (TURN && kind != 1 && turned) {
        float b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = HALF ? (float)other.x[e] : a[e ^ 1];
        if (kind == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const double2 z = cs[e * LPH + x];
            b[e] = (float)__builtin_fma((double)a[e], z.x, (double)b[e] * z.y);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 z = cs_q[e * LPH + x];
            b[e] = __builtin_fmaf(a[e], z.x, b[e] * z.y);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * x + e < P.rot) a[e] = b[e];  // (the others as they were: a factor of zero may have an infinity beside it)
      }
      if (kind == 2) {
        if (there) store8((T*)P.q_out + (tok * P.Hq + g) * D + 8 * x, a);
        mine = next;
        other = next_other;
        continue;
      }
      // (all lanes take part in what follows)
      unsigned largest = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(a[e]) & 0x7fffffffu);
      largest = max(largest, (unsigned)__builtin_amdgcn_update_dpp(0, (int)largest, 0xb1, 0xf, 0xf, false));  // lanes 1, 0, 3, 2 of four
      largest = max(largest, (unsigned)__builtin_amdgcn_update_dpp(0, (int)largest, 0x4e, 0xf, 0xf, false));  // 2, 3, 0, 1
      const unsigned bits = step_of(largest);
      const float step = __uint_as_float(bits);
      unsigned word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) word |= code_of(a[e], step) << 4 * e;
      if (!(step > 0.f)) word = 0;
      const int64_t row = row0 + (int64_t)g * P.cache.page_size;
      const bool kept = there && row0 >= 0;
      if (kept && x % 4 == 0) ((unsigned short*)(kind == 0 ? P.cache.k_step : P.cache.v_step))[row * (D / 32) + x / 4] = (unsigned short)(bits >> 16);
      if (kind == 0) {
        if (kept) *(unsigned*)(P.cache.k + row * (D / 2) + (x % 4) * (D / 8) + 4 * (x / 4)) = word;
      } else {  // word i of 16, the head's lanes two (D = 64: half) a word
        codes[wave][lane] = word;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int w16 = 0; w16 < 16; w16 += LPH) {
          const int i16 = w16 + x;
          unsigned w = 0;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) w |= (codes[wave][sub * LPH + 2 * j + (i16 >> 3)] >> 4 * (i16 & 7) & 15u) << 4 * j;
          if (!kept) continue;
          if (D == 128) *(unsigned*)(P.cache.v + row * (D / 2) + 4 * i16) = w;
          else *(unsigned short*)(P.cache.v + row * (D / 2) + 2 * i16) = (unsigned short)w;
        }
        asm volatile("" ::: "memory");
      }
      T* const held = (T*)(kind == 0 ? P.k_held : P.v_held);
      if (held && there) {
        float y[8];
        auto put = [&](auto sel) __attribute__((always_inline)) {
          constexpr int SEL = decltype(sel)::value;
          typedef float f32x2 __attribute__((ext_vector_type(2)));
          const f32x2 z = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, SEL);
          y[2 * SEL] = z[0] * step;
          y[2 * SEL + 1] = z[1] * step;
        };
        put(std::integral_constant<int, 0>()); put(std::integral_constant<int, 1>()); put(std::integral_constant<int, 2>()); put(std::integral_constant<int, 3>());
        store8(held + (tok * P.Hkv + g) * D + 8 * x, y);
      }
      mine = next;
      other = next_other;
    }
    asm volatile("" ::: "memory");
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
  if (!aligned16(q_out) || !aligned16(k_held) || !aligned16(v_held) || !aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_step) || !aligned16(c->v_step)) {
    set_error("a buffer does not start at a multiple of 16 bytes");
    return SB_ERR_INVALID_ARG;
  }
  // (several lanes read what one of them overwrites, and tokens are at work side by side)
  const int64_t esize = c->dtype == SB_F32 ? 4 : 2;
  struct Range { const char* at; int64_t bytes; };
  auto range = [&](const void* at, int H, int64_t pitch) { return Range{(const char*)at, at ? ((n->total_new - 1) * pitch + (int64_t)H * D) * esize : 0}; };
  const Range read[] = {range(q, Hq, q_pitch), range(k, Hkv, k_pitch), range(v, Hkv, v_pitch)};
  const Range written[] = {range(q_out, Hq, (int64_t)Hq * D), range(k_held, Hkv, (int64_t)Hkv * D), range(v_held, Hkv, (int64_t)Hkv * D)};
  auto meet = [](const Range& a, const Range& b) { return a.bytes > 0 && b.bytes > 0 && (uintptr_t)a.at < (uintptr_t)b.at + b.bytes && (uintptr_t)b.at < (uintptr_t)a.at + a.bytes; };
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 3; ++j)
      if (meet(written[i], read[j]) || (i < j && meet(written[i], written[j]))) {
        set_error("outputs in the place of inputs or of each other are not supported");
        return SB_ERR_INVALID_ARG;
      }
  const int64_t rows = (int64_t)c->num_pages * Hkv * c->page_size;
  const Range others[] = {{(const char*)c->k, rows * (D / 2)}, {(const char*)c->v, rows * (D / 2)}, {(const char*)c->k_step, rows * (D / 16)}, {(const char*)c->v_step, rows * (D / 16)},
                          {(const char*)c->page_table, (int64_t)n->num_seqs * c->max_pages * 4}, {(const char*)n->cu_new, ((int64_t)n->num_seqs + 1) * 4},
                          {(const char*)n->cached, (int64_t)n->num_seqs * 4}, {(const char*)positions, positions ? (int64_t)axes->num_axes * n->total_new * 4 : 0}};
  for (const Range& w : written)
    for (const Range& x : others)
      if (meet(w, x)) { set_error("outputs in the place of the pages, their table, positions, cu_new or cached are not supported"); return SB_ERR_INVALID_ARG; }
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
  const bool wide = aligned16(q) && aligned16(k) && aligned16(v) && q_pitch * esize % 16 == 0 && k_pitch * esize % 16 == 0 && v_pitch * esize % 16 == 0 &&
                    (!r || r->layout != SB_ROPE_HALF || r->rot_dim % 16 == 0);
  // Four wavefronts to a token where tokens are few; where they fill the chip, one, which looks up and computes what a token has once.
  // (32/8 heads, one and four, in us: 512 tokens 15.0 and 13.7, 1536 17.9 and 14.9, 2048 18.2 both, 4096 24.4 and 29.0, 8192 42.0 and 47.2)
  P.waves = P.T < 2048 ? 4 : 1;
  // A token each: 4096 wavefronts fill the chip, and those behind them start as others end.  Two, where all are there at once and take 15/16 of that or more: then nobody starts twice.  (In float32,
  // where a token is twice the bytes, never.)  32/8 heads, one and two each, in us: 4600 tokens 33.3 and 39.4, 6500 42.6 and 44.7, 7500 46.1 both, 8000 47.1 and 46.6, 8192 47.6 and 46.8, 8300 54.2 and 63.5, 10000 62.0
  // and 71.2, 16384 95.5 and 99.7;  8 heads of 128 8192 28.1 and 26.9, 8300 30.4 and 34.6;  14/2 of 64 19.8 and 19.0, 21.7 and 23.9;  float32 8192 87.1 and 95.4.  Four: 8192 66.5, 32768 186 (one 183)
  P.run = esize == 2 && P.T <= 8192 && P.T > 8192 / 16 * 15 ? 2 : 1;
  if (P.T >> 25 > P.run) P.run = P.T >> 25;  // (a launch has fewer than 2^32 threads)
  const int64_t per = (int64_t)P.run * 4 / P.waves;
  const dim3 grid((unsigned)((P.T + per - 1) / per));
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
