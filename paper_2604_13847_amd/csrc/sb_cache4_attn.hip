// Attention of new tokens over a paged cache in four bits (serving).
//
//   S_tu = scale sum_c step_uc (sum over d in group c of q_td n_ud),   O_td = sum_u (P_tu step_uc) m_ud   (c: d's group)
//
// n and m, the levels of keys and values, are exact as operands of matrix instructions; steps are applied in float32, to the scores of a group's product and to the probabilities.
//
// Few new tokens (cache4_split_kernel): bound by the cache's bytes, 72 a token and KV head each for K and V at head_dim 128.  64 sequences of 500 to 32768 tokens, 32/8 heads: 130 us with
// the join, 4.4 TB/s (such bytes at the rate of a copy: 113); head_dim 64: 76 (57), where the arithmetic of a strip is not all hidden.  More rows are bound by it: 8 sequences of 20000, 16 rows a KV head 55 us, 32 73, 64
// 111 (37; vector instructions 67 % of the cycles at 64).  One of 4097: 14.1 us, 9.8 and 3.5 of its two launches, each a chain of dependent loads.  In float32
// each product is three of bfloat16.
// Many (cache4_chunk_kernel, cache4_chunk_stream_kernel): bound by the matrix and vector instructions of a tile.  2 x 2000 tokens behind 20000 and 30001, window 8192, 28/4 heads: 483 us,
// 914 TFLOP/s; a prompt of 6001, 32/8 heads: 334 us, 0.88 PFLOP/s.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sb_cache4.h"
#include "sb_window_fwd.h"

// x y, and 0 where either is 0, whatever the other is (v_mul_legacy_f32: as fast as the other product, subnormal numbers alike)
extern "C" __device__ float zero_product(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

namespace sb {

struct CutItem {  // an item that a workgroup has the first part of
  int row0, rows, m0, g;  // its sequence's first packed row and flattened rows, its own first, its KV head
  int parts, reserved[3];
};
struct Cache4Params {
  WindowParams w;  // (of its cache, the page table alone is read)
  PagedCache4 cache;
  int unit;  // see Stream
  CutItem* cuts;  // of every workgroup
};

typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// byte SEL of x, two levels, as bfloat16: lower half first
template <int SEL> __device__ inline bf16x2 levels(unsigned x) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, 1.0f, SEL); }
__device__ inline bf16x8 levels8(unsigned x) {
  const bf16x2 a = levels<0>(x), b = levels<1>(x), c = levels<2>(x), d = levels<3>(x);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ inline Rsrc resource(const void* base, unsigned bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x20000); }
// Eight numbers as PIECES bfloat16 numbers each: one, rounded, or three of eight significant bits that add up to it.
template <int PIECES> __device__ __attribute__((always_inline)) inline void pieces_of(const float (&x)[8], bf16x8 (&to)[PIECES]) {
  if constexpr (PIECES == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) to[0][e] = (bf16)x[e];
  } else {
    u32x4 y[PIECES];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float a = x[2 * e], b = x[2 * e + 1];
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        y[p][e] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);  // their upper halves
        a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
      }
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) to[p] = __builtin_bit_cast(bf16x8, y[p]);
  }
}
template <int SEL> __device__ inline f32x2 numbers(unsigned x) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, 1.0f, SEL); }
__device__ inline float step_at(unsigned pair, int i) { return __uint_as_float(i & 1 ? pair & 0xffff0000u : pair << 16); }

// Matrix instructions 16x16x32 over a strip of 32 keys: lane = (l16, qd).
//   scores S^T = K Q^T: A row = key 16 b + l16, slots of quarter qd = elements 32 c + 8 qd + (0 .. 7); C row 4 qd + v = key 16 b + 4 qd + v, column l16
//   output O^T += V^T P^T: slot j of quarter qd = key 16 (j / 4) + 4 qd + j % 4, which is where the scores are; A row = element 16 t + l16 of tile t
// A tile of R = 16 / PARTS rows takes all 16 columns: row l16 / PARTS, PARTS times, each time for GROUPS / PARTS of the groups of 32 elements.  A column's query is zero in the groups
// that are not its own, so that one chain of products leaves every column with its own group's share of the score, to be multiplied by that group's step and added up over
// the columns of a row; and the probabilities that it multiplies with its own group's steps are right for that group's tiles of the output, the others of which are not used.
// So four rows (a token of four heads) cost a step's multiplication once and not four times.
// A strip on its way: a wavefront's own place in LDS, filled by asynchronous loads of 16 bytes (codes) and 4 bytes (steps) a lane, each lane's bytes behind the lane's before it.
//   head_dim 128: K in two loads of 16 rows, 16-byte piece b of row r at 4 r + (b ^ r / 4), so that the 16 rows of an operand lie in different banks; V likewise, row r at
//   16 (r % 4) + 4 (r / 4), so that the four rows that a slot's quarters read lie side by side; the steps of K, and of V, in one load of 32 rows each
//   head_dim 64: K and V in one load of 32 rows each, in order; the steps of both in one
template <int D>
struct StripLoader {
  static constexpr int LOADS = D == 128 ? 6 : 3, CODES = 32 * D / 2, STEPS = 32 * D / 16, BYTES = 2 * CODES + 2 * STEPS;
  unsigned k_at, v_at, step_at_;  // bytes from the first row of the lane's 16 to what the lane loads
  bool upper;                     // the lane's rows are the strip's second 16 (head_dim 128: of the steps)
  __device__ inline void init(int lane) {
    if constexpr (D == 128) {
      const int r = lane >> 2, r_v = (r & 3) * 4 + (r >> 2);
      k_at = r * 64 + 16 * ((lane & 3) ^ (r >> 2));
      v_at = r_v * 64 + 16 * (lane & 3);
      step_at_ = (lane & 31) * 4;
    } else {
      k_at = v_at = (lane & 31) * 16;
      step_at_ = (lane & 15) * 4;
    }
    upper = lane >= 32;
  }
  static __device__ __attribute__((always_inline)) inline void issue16(unsigned off, const void* base, unsigned slot) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %2" : : "v"(off), "s"(slot), "s"(base) : "memory", "m0");
  }
  static __device__ __attribute__((always_inline)) inline void issue16(const void* from, unsigned slot) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(slot) : "memory", "m0");
  }
  static __device__ __attribute__((always_inline)) inline void issue4(const void* from, unsigned slot) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dword %0, off" : : "v"(from), "s"(slot) : "memory", "m0");
  }
  // row0, row1: first rows of the strip's two 16 in the cache's arrays; slot: where in LDS (both wave-uniform)
  __device__ __attribute__((always_inline)) inline void issue(const PagedCache4& c, uint64_t row0, uint64_t row1, unsigned slot, int lane) const {
    if constexpr (D == 128) {
      issue16(k_at, c.k + row0 * 64, slot);
      issue16(k_at, c.k + row1 * 64, slot + CODES / 2);
      issue16(v_at, c.v + row0 * 64, slot + CODES);
      issue16(v_at, c.v + row1 * 64, slot + CODES + CODES / 2);
      const uint64_t at = (upper ? row1 : row0) * 8 + step_at_;
      issue4((const char*)c.k_step + at, slot + 2 * CODES);
      issue4((const char*)c.v_step + at, slot + 2 * CODES + STEPS);
    } else {
      const uint64_t at = (upper ? row1 : row0) * 32 + k_at;
      issue16(c.k + at, slot);
      issue16(c.v + at, slot + CODES);
      issue4((const char*)(upper ? c.v_step : c.k_step) + ((lane & 16) ? row1 : row0) * 4 + step_at_, slot + 2 * CODES);
    }
  }
};
// What a lane reads of a strip.  OWN: the lane's own groups, part OWN + (0 .. OWN - 1).
template <int D, int OWN>
struct StripReader {
  static constexpr int GROUPS = D / 32, CODES = StripLoader<D>::CODES, STEPS = StripLoader<D>::STEPS;
  unsigned k_at, v_at, s_at;
  unsigned mine;  // OWN == 1: the bytes of the lane's own step, of a key's (zeros below them); OWN == 2: which half of them
  __device__ inline void init(int l16, int qd, int part) {
    if constexpr (D == 128) {
      k_at = l16 * 64 + 16 * (qd ^ (l16 >> 2));
      v_at = CODES + qd * 64 + l16 * 4;  // row 4 qd + j: at 64 (4 j + qd)
    } else {
      k_at = l16 * 32 + qd * 8;
      v_at = CODES + qd * 128 + l16 * 2;
    }
    s_at = 2 * CODES + qd * 4 * GROUPS * 2;
    mine = OWN == 1 ? 0x01000c0cu + 0x02020000u * part : part;
  }
  template <typename V> static __device__ __attribute__((always_inline)) inline V at(unsigned a) { return *(const V __attribute__((address_space(3)))*)(uintptr_t)a; }
  __device__ __attribute__((always_inline)) inline void keys(unsigned (&k)[2][GROUPS], unsigned slot) const {  // [b][c]
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      typedef typename std::conditional<D == 128, u32x4, u32x2>::type Piece;
      const Piece y = at<Piece>(slot + k_at + b * (CODES / 2));
#pragma unroll
      for (int c = 0; c < GROUPS; ++c) k[b][c] = y[c];
    }
  }
  // Word l16 of slot j's key (head_dim 64: 16 bits).  v: those of slots 0, 1, .. 7 (head_dim 64: of 0 and 2, 1 and 3, 4 and 6, 5 and 7)
  static constexpr int WORDS = D / 16;
  __device__ __attribute__((always_inline)) inline void values(unsigned (&v)[WORDS], unsigned slot) const {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < WORDS / 2; ++j) {
        const unsigned from = slot + v_at + b * (CODES / 2);
        if constexpr (D == 128) v[4 * b + j] = at<unsigned>(from + 256 * j);
        else v[2 * b + j] = __builtin_bit_cast(unsigned, u16x2{at<unsigned short>(from + 32 * j), at<unsigned short>(from + 32 * (j + 2))});
      }
  }
  // of keys 16 b + 4 qd + v: steps of the lane's own groups.  16 bytes at a time, all groups', of which a lane keeps its own
  __device__ __attribute__((always_inline)) inline void steps(float (&to)[2][4][OWN], unsigned slot, bool of_values) const {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const unsigned from = slot + s_at + (of_values ? STEPS : 0) + b * (STEPS / 2);
      unsigned x[2 * GROUPS];
#pragma unroll
      for (int i = 0; i < GROUPS / 2; ++i) {
        const u32x4 y = at<u32x4>(from + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const unsigned* const of = x + v * GROUPS / 2;  // key v's
        if constexpr (OWN == 1) {
          to[b][v][0] = __uint_as_float(__builtin_amdgcn_perm(of[GROUPS / 2 - 1], of[0], mine));
        } else if constexpr (OWN == GROUPS) {
#pragma unroll
          for (int o = 0; o < OWN; ++o) to[b][v][o] = step_at(of[o / 2], o);
        } else {
          static_assert(OWN == 2 && GROUPS == 4, "a lane's own two groups are a word");
          const unsigned y = mine ? of[1] : of[0];
          to[b][v][0] = step_at(y, 0);
          to[b][v][1] = step_at(y, 1);
        }
      }
    }
  }
};
// over the columns of a row: lanes that differ in the lowest bits.  The same in all of them, bit for bit: columns that disagreed about the maximum of their row would be relative to different
// references.  So x is rounded first: as a sum of products, of which one is rounded and the other is not, it would depend on whose is the lane's own.
template <int PARTS> __device__ inline float add_parts(float x) {
  if constexpr (PARTS > 1) asm("" : "+v"(x));
  auto swapped = [](float y, auto ctrl) { return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(y), decltype(ctrl)::value, 0xf, 0xf, true)); };  // (so written, it becomes part of the sum)
  if constexpr (PARTS >= 2) x += swapped(x, std::integral_constant<int, 0xb1>());  // 1, 0, 3, 2
  if constexpr (PARTS >= 4) x += swapped(x, std::integral_constant<int, 0x4e>());  // 2, 3, 0, 1
  if constexpr (PARTS > 1) asm("" : "+v"(x));  // (moved behind a branch, the sum would not be one instruction)
  return x;
}

// The work as one stream of strips (of TILE keys): sequence by sequence, KV head by head, tile of rows by tile, as many strips as any tile of the sequence has.  (A tile's own are the
// first of these.)  Every workgroup takes as many neighbouring strips as the others, whatever the lengths, which only the device knows; where that
// cuts an item, its parts are joined by a launch that follows.  Only a workgroup's first and last items can be cut, so two places a workgroup hold all parts.
// Counted in units of 2^unit strips, so that 31 bits hold the stream.  Where P.splits is 1, an item counts as one unit, and a workgroup has whole items.
// (64 sequences of 500 to 32768 tokens, before the strips went through LDS: items of 2048 keys, whose number goes by the longest sequence, left 3 of 4 workgroups without work: 175 us, 155 as a stream.)
struct Item {
  RowTile t;
  int g;
  int first, count;  // units of the stream
};
template <int ROWS, int TILE>
struct Stream {
  int row0, n, pos0, tiles, count;  // of sequence base + lane
  __device__ inline int size(const WindowParams& P) const { return tiles * count * P.Hkv; }
  struct Lengths { int from, to, cached; };  // as they are in memory
  static __device__ inline Lengths fetch(const Cache4Params& A, int base, int lane) {
    const int s = base + lane;
    return (unsigned)s < (unsigned)A.w.S ? Lengths{A.w.cu[s], A.w.cu[s + 1], A.w.cached[s]} : Lengths{};
  }
  __device__ inline void take(const Cache4Params& A, const Lengths& x, int base, int lane) {
    const WindowParams& P = A.w;
    row0 = n = pos0 = tiles = count = 0;
    if (base + lane < P.S) {
      row0 = x.from;
      n = x.to;
      pos0 = x.cached;
      row0 = min(max(row0, 0), P.T);
      n = min(max(min(n, P.T) - row0, 0), P.max_new);
      if (n * P.G < P.rows_from || n * P.G > P.rows_to) n = 0;
      pos0 = min(max(pos0, 0), 0x7fffffff - n);
    }
    if (n > 0) {
      tiles = (int)(((unsigned)n * (unsigned)P.G + (unsigned)ROWS - 1) / (unsigned)ROWS);
      count = KeyTiles<TILE>(pos0, min(pos0 + n - 1, P.cache.max_pages * P.cache.page_size - 1), P.window, P.sinks).count();
      // and no more than fit the window of a tile's rows (of `length` tokens and keys in a row, at most) and the sinks
      const int64_t length = (int64_t)P.window + (ROWS + P.G - 2) / P.G;
      count = (int)min((int64_t)count, (length + TILE - 2) / TILE + 1 + ((int64_t)P.sinks + TILE - 1) / TILE);
      count = P.splits == 1 ? 1 : max((count + (1 << A.unit) - 1) >> A.unit, 1);  // (rows that see nothing have a result too)
    }
  }
  // units of a workgroup.  With up to 64 sequences, these stay loaded.  (600 sequences of 100 to 500 tokens: 79 us with every 64 loaded when it was their turn, 64 so.)
  __device__ inline int share(const Cache4Params& A, int workgroups, int least, int lane) {
    Lengths next = fetch(A, 0, lane);
    if (A.w.splits == 1) {
      if (A.w.S <= 64) take(A, next, 0, lane);
      return 1;
    }
    int sum = 0;
    for (int base = 0; base < A.w.S; base += 64) {
      const Lengths x = next;
      if (base + 64 < A.w.S) next = fetch(A, base + 64, lane);  // (on its way while these are worked on)
      take(A, x, base, lane);
      sum += size(A.w);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
      if (off < A.w.S) sum += __shfl_xor(sum, off, 64);
    const unsigned all = (unsigned)__builtin_amdgcn_readfirstlane(sum), each = (all + (unsigned)workgroups - 1) / (unsigned)workgroups;
    return __builtin_amdgcn_readfirstlane((int)((each + (unsigned)least - 1) / (unsigned)least * (unsigned)least));
  }
  // The sequence that the last item found was of: where it is among the stream's units, its tiles and units of each, and the 64 that it was loaded with.  (Wave-uniform.  Its other items are
  // found without a load, and the next sequence from there on: 600 sequences of 100 to 8000 478 -> 350 us.)
  RowTile seq;
  int start, end, seq_tiles, seq_count, base, before;
  // the item that unit x belongs to; s < 0: there are no so many.  first: nothing was asked before, and up to 64 sequences are loaded; else x is no less than the last one
  __device__ inline Item find(const Cache4Params& A, int x, int lane, bool first) {
    const WindowParams& P = A.w;
    Item r{};
    r.t.s = -1;
    if (first) base = before = end = 0;
    if (first || x >= end) {
      const bool loaded = first && P.S <= 64;
      Lengths next{};
      if (!loaded) next = fetch(A, base, lane);
      for (; base < P.S; base += 64) {
        if (!loaded) {
          const Lengths here = next;
          next = fetch(A, base + 64, lane);
          take(A, here, base, lane);
        }
        const int mine = size(P);
        int incl = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1)
          if (off < P.S - base) {
            const int y = __shfl_up(incl, off, 64);
            if (lane >= off) incl += y;
          }
        const unsigned long long hit = __builtin_amdgcn_ballot_w64(base + lane < P.S && x - before < incl);
        if (hit) {
          const int src = __builtin_ctzll(hit);
          seq = RowTile{base + src, 0, __builtin_amdgcn_readlane(row0, src), __builtin_amdgcn_readlane(n, src), __builtin_amdgcn_readlane(pos0, src)};
          seq_tiles = __builtin_amdgcn_readlane(tiles, src);
          seq_count = __builtin_amdgcn_readlane(count, src);
          start = before + __builtin_amdgcn_readlane(incl - mine, src);
          end = before + __builtin_amdgcn_readlane(incl, src);
          break;
        }
        before += __builtin_amdgcn_readlane(incl, min(P.S - base, 64) - 1);
      }
      if (base >= P.S) return r;
    }
    const unsigned item = (unsigned)(x - start) / (unsigned)seq_count, g = item / (unsigned)seq_tiles;
    r.count = seq_count;
    r.first = __builtin_amdgcn_readfirstlane(start + (int)item * seq_count);
    r.g = __builtin_amdgcn_readfirstlane((int)g);
    r.t = seq;
    r.t.tile = __builtin_amdgcn_readfirstlane((int)(item - g * (unsigned)seq_tiles));
    return r;
  }
};

// Parts of a cut item that begins in this workgroup and has the stream's unit `last`.  (No more than there are workgroups from here on, whatever cu_new says.)
__device__ inline int parts_of(int last, int share) { return (int)min((unsigned)last / (unsigned)share, gridDim.x - 1) - (int)blockIdx.x + 1; }

// An item is up to 16 NT / PARTS flattened rows of a KV head; a wavefront takes every NW-th of the workgroup's strips of it through its own ring in LDS, without any barrier, the next ones on their
// way while one is worked on.  PIECES: a query and a probability as that many bfloat16 numbers.
constexpr int kWaves4 = 4;
// Wavefronts of a SIMD, as many as the registers of a strip's numbers allow, and stages of a ring, so that the rings of as many workgroups fit a CU: what a strip takes is one product, sum and
// exponential after the other, which other wavefronts have to fill.  64 sequences of 500 to 32768 tokens, 32/8 heads, with one wavefront less and with these: head_dim 128 134 and 130 us,
// head_dim 64 84 and 78 (and with one more, which spills, 102); float32, 28/4 heads, 500 to 8000: 47 and 42.
constexpr int split_waves(int D, int rows, int pieces) {
  if (D == 64) return pieces == 3 ? (rows == 8 ? 4 : 3) : rows == 8 ? 5 : rows == 16 ? 4 : 2;
  return rows == 4 && pieces == 1 ? 4 : rows <= 8 ? 3 : 2;
}
constexpr int split_stages(int D, int rows, int pieces) { return split_waves(D, rows, pieces) >= (D == 64 ? 5 : 3) ? 2 : 4; }
template <typename T, int D, int PARTS, int NT, int PIECES>
__global__ __launch_bounds__(64 * kWaves4) __attribute__((amdgpu_waves_per_eu(split_waves(D, 16 * NT / PARTS, PIECES)))) void cache4_split_kernel(Cache4Params A) {
  const WindowParams& P = A.w;
  constexpr int NW = kWaves4, R = 16 / PARTS, ROWS = R * NT, GROUPS = D / 32, OWN = GROUPS / PARTS, TILES = D / 16;
  static_assert(OWN * PARTS == GROUPS, "every column has groups of its own");
  constexpr int OUT_P = D + 4;  // floats from row to row of a wavefront's sums in LDS
  constexpr int STAGES = split_stages(D, ROWS, PIECES), LOADS = StripLoader<D>::LOADS, SLOT = StripLoader<D>::BYTES;
  constexpr float kLazy = 8.0f;
  __shared__ __attribute__((aligned(1024))) char ring[NW][STAGES * SLOT];
  static_assert(ROWS * OUT_P * 4 <= STAGES * SLOT && STAGES * SLOT % 16 == 0, "the sums take the strips' place");
  __shared__ float stats[2][NW][ROWS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, qd = lane >> 4;
  const int part = l16 % PARTS, r16 = l16 / PARTS;
  const unsigned ring0 = __builtin_amdgcn_readfirstlane((int)lds_offset(ring[wave]));
  StripLoader<D> loader;
  loader.init(lane);
  StripReader<D, OWN> reader;
  reader.init(l16, qd, part);
  Stream<ROWS, 32> stream;
  const int share = stream.share(A, gridDim.x, NW >> A.unit > 0 ? NW >> A.unit : 1, lane);
  const int64_t x_last = (int64_t)share * (blockIdx.x + 1);
  int x_first = (int)min(x_last - share, (int64_t)0x7fffffff);  // (the stream ends before)
  const int x_end = (int)min(x_last, (int64_t)0x7fffffff);
  Item item = stream.find(A, x_first, lane, true);
  CutItem cut{};
  while (item.t.s >= 0) {
    const RowTile t = item.t;
    const int g = item.g, x_next = min(x_end, item.first + item.count);
    const int rows = t.n * P.G, m0 = t.tile * ROWS, mine = min(rows - m0, ROWS);
    auto token = [&](int m) { return (int)((unsigned)min(m, rows - 1) / (unsigned)P.G); };
    const int ta = __builtin_amdgcn_readfirstlane(t.pos0 + token(m0)), last = __builtin_amdgcn_readfirstlane(t.pos0 + token(m0 + ROWS - 1));
    const int tb = min(last, A.cache.max_pages * A.cache.page_size - 1), end = tb + 1, lo = max(0, ta - P.window + 1);
    const KeyTiles<32> strips(ta, tb, P.window, P.sinks);
    const int begin = (int)min((int64_t)(x_first - item.first) << A.unit, (int64_t)strips.count());
    const int count = P.splits == 1 ? strips.count() : (int)min((int64_t)(x_next - item.first) << A.unit, (int64_t)strips.count());
    const bool whole = x_first == item.first && x_next == item.first + item.count;
    const int turns = A.cache.num_pages == 0 ? 0 : max(count - begin - wave + NW - 1, 0) / NW;  // strips of this wavefront: begin + wave + NW x (may be none)
    const int32_t* const table = A.cache.table + (int64_t)t.s * A.cache.max_pages;

    // Of strip begin + wave + NW (x0 + lane): the page of its keys 0 .. 15 and 16 .. 31, and how many of each exist.  (Where none does, page 0 stands in: its rows are read and not used.)
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
            const int page = table[u >> A.cache.page_shift];
            if ((unsigned)page < (unsigned)A.cache.num_pages) {
              there[b] = min(end - u, 16);
              where[b] = page;
            }
          }
        }
      }
    };
    auto issue = [&](int x) __attribute__((always_inline)) {  // strip x of this wavefront
      const int u = __builtin_amdgcn_readfirstlane(32 * strips.at(begin + wave + NW * x));
      uint64_t row[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const unsigned page = (unsigned)__builtin_amdgcn_readlane(where[b], x - x0);
        // (16 rows of a page, all of them in memory, whether or not they have been written)
        row[b] = ((uint64_t)(page * (uint64_t)A.cache.Hkv + g) << A.cache.page_shift) + ((u + 16 * b) & (A.cache.page_size - 1));
      }
      loader.issue(A.cache, row[0], row[1], ring0 + (x & (STAGES - 1)) * SLOT, lane);
    };

    look_up(0);  // (on its way beside the queries)

    // B operand of the scores: column = row r16 of tile nt, zero in groups that are not the column's own
    bf16x8 qf[NT][GROUPS][PIECES];
    int pos[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int m = min(m0 + R * nt + r16, rows - 1), i = token(m), h = g * P.G + m - i * P.G;
      pos[nt] = t.pos0 + i;
      const T* const q = (const T*)P.q + ((int64_t)(t.row0 + i) * P.Hq + h) * D + 8 * qd;
#pragma unroll
      for (int c = 0; c < GROUPS; ++c) {
        if constexpr (PIECES == 1) {
          qf[nt][c][0] = *(const bf16x8*)(q + 32 * c);
        } else {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = (float)q[32 * c + e];
          pieces_of<PIECES>(y, qf[nt][c]);
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
          if (PARTS > 1 && part != c / OWN) qf[nt][c][p] = zero_bf16x8();
      }
    }
    f32x4 acc[NT][TILES];
    float top[NT], neg[NT], l[NT];  // the reference of the exponentials (a score, and what is added to them), this lane's share of their sum
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int d = 0; d < TILES; ++d) acc[nt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      top[nt] = -__builtin_inff();
      neg[nt] = 0.f;
      l[nt] = 0.f;
    }

    auto work = [&](int x) __attribute__((always_inline)) {
      const unsigned slot = ring0 + (x & (STAGES - 1)) * SLOT;
      constexpr int WORDS = StripReader<D, OWN>::WORDS;
      unsigned keys[2][GROUPS], values[WORDS];
      float k_step[2][4][OWN], v_step[2][4][OWN];
      reader.keys(keys, slot);
      reader.steps(k_step, slot, false);
      const int u0 = __builtin_amdgcn_readfirstlane(32 * strips.at(begin + wave + NW * x));
      const unsigned have = (1u << __builtin_amdgcn_readlane(there[0], x - x0)) - 1 | ((1u << __builtin_amdgcn_readlane(there[1], x - x0)) - 1) << 16;  // keys that exist
      float sc[NT][2][4];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x4 y[NT][OWN];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int o = 0; o < OWN; ++o) y[nt][o] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < GROUPS; ++c) {
          const bf16x8 op = levels8(keys[b][c]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int p = PIECES - 1; p >= 0; --p) y[nt][c % OWN] = mfma16(op, qf[nt][c][p], y[nt][c % OWN]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            float z = y[nt][0][v] * k_step[b][v][0];
#pragma unroll
            for (int o = 1; o < OWN; ++o) z = __builtin_fmaf(y[nt][o][v], k_step[b][v][o], z);
            sc[nt][b][v] = add_parts<PARTS>(z);
          }
      }
      if constexpr (NT > 1) __builtin_amdgcn_sched_barrier(0);
      reader.values(values, slot);
      reader.steps(v_step, slot, true);
      if (u0 + 31 > ta || (last - u0 >= P.window && u0 + 31 >= P.sinks) || have != ~0u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int r = 16 * b + 4 * qd + v;
              if (!sees(pos[nt], u0 + r, P.window, P.sinks) || !(have >> r & 1)) sc[nt][b][v] = -__builtin_inff();
            }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float mx = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sc[nt][b][v]);
        // running maximum, followed lazily: the reference moves only when a score exceeds it by 2^kLazy
        if (__builtin_amdgcn_ballot_w64(!((mx - top[nt]) * P.scale_log2e <= kLazy)) != 0) {
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          const bool first = top[nt] == -__builtin_inff();  // nothing accumulated yet for this row
          const bool move = first | ((mx - top[nt]) * P.scale_log2e > kLazy);
          const float now = move ? fmaxf(top[nt], mx) : top[nt];
          const float use = now == -__builtin_inff() ? 0.f : now;  // no key seen yet: keep the exponent finite
          const float alpha = first ? 1.0f : fast_exp2((top[nt] - use) * P.scale_log2e);
          neg[nt] = -use * P.scale_log2e;
          top[nt] = now;
          if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
            l[nt] *= alpha;
#pragma unroll
            for (int d = 0; d < TILES; ++d)
#pragma unroll
              for (int v = 0; v < 4; ++v) acc[nt][d][v] *= alpha;
          }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            sc[nt][b][v] = fast_exp2(__builtin_fmaf(sc[nt][b][v], P.scale_log2e, neg[nt]));
            l[nt] += sc[nt][b][v];
          }
      }
      // levels of two keys side by side in a byte: even and odd tiles' (a word's nibble t is element 16 t + l16)
      unsigned even[WORDS / 2], odd[WORDS / 2];
#pragma unroll
      for (int j = 0; j < WORDS / 2; ++j) {
        const unsigned a = values[2 * j], b = values[2 * j + 1];
        even[j] = (a & 0x0f0f0f0fu) | (b << 4 & 0xf0f0f0f0u);
        odd[j] = (a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u);
      }
      bf16x8 w[NT][PIECES];
      // Probabilities times the steps of one of the lane's groups.  Where a key is hidden from a row, or does not exist, the probability is 0, and whatever step it has, a NaN too, reaches nothing.
      auto weights = [&](auto oc) __attribute__((always_inline)) {
        constexpr int O = decltype(oc)::value;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = zero_product(sc[nt][j / 4][j % 4], v_step[j / 4][j % 4][O]);
          pieces_of<PIECES>(y, w[nt]);
        }
      };
      auto tile = [&](auto tc) __attribute__((always_inline)) {
        constexpr int TT = decltype(tc)::value;
        bf16x8 op;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned from = TT & 1 ? odd[j * WORDS / 8] : even[j * WORDS / 8];
          const bf16x2 y = D == 128 || j % 2 == 0 ? levels<TT / 2>(from) : levels<(TT / 2 + 2) % 4>(from);
          op[2 * j] = y[0];
          op[2 * j + 1] = y[1];
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int p = PIECES - 1; p >= 0; --p) acc[nt][TT] = mfma16(op, w[nt][p], acc[nt][TT]);
      };
      auto group = [&](auto oc) __attribute__((always_inline)) {  // groups O, O + OWN, ..: two tiles each
        constexpr int O = decltype(oc)::value;
        if constexpr (NT > 1) __builtin_amdgcn_sched_barrier(0);  // (one group's numbers at a time: all of them spill)
        weights(oc);
        tile(std::integral_constant<int, 2 * O>());
        tile(std::integral_constant<int, 2 * O + 1>());
        if constexpr (O + OWN < GROUPS) { tile(std::integral_constant<int, 2 * (O + OWN)>()); tile(std::integral_constant<int, 2 * (O + OWN) + 1>()); }
        if constexpr (O + 2 * OWN < GROUPS) { tile(std::integral_constant<int, 2 * (O + 2 * OWN)>()); tile(std::integral_constant<int, 2 * (O + 2 * OWN) + 1>()); }
        if constexpr (O + 3 * OWN < GROUPS) { tile(std::integral_constant<int, 2 * (O + 3 * OWN)>()); tile(std::integral_constant<int, 2 * (O + 3 * OWN) + 1>()); }
      };
      group(std::integral_constant<int, 0>());
      if constexpr (OWN > 1) group(std::integral_constant<int, 1>());
      if constexpr (OWN > 2) { group(std::integral_constant<int, 2>()); group(std::integral_constant<int, 3>()); }
    };

    // the query operands must have landed before the strips' loads start: from there on only those are in flight, and waited for by hand
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < GROUPS; ++c)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) asm volatile("" : "+v"(qf[nt][c][p]));
    for (int from = 0; from < turns; from += 64) {  // (a look-up's worth)
      const int to = min(from + 64, turns);
      if (from > 0) look_up(from);
      asm volatile("s_waitcnt vmcnt(0)" : "+v"(where[0]), "+v"(where[1]), "+v"(there[0]), "+v"(there[1]) : : "memory");
#pragma unroll
      for (int i = 0; i < STAGES - 1; ++i)
        if (from + i < to) issue(from + i);
      for (int x = from; x < to; ++x) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the strip before has been read: its place is free
        if (x + STAGES - 1 < to) issue(x + STAGES - 1);
        const int behind = to - 1 - x;  // strips on their way behind this one
        if (STAGES == 4 && behind >= 3) wait_vmcnt<3 * LOADS>();
        else if (STAGES == 4 && behind == 2) wait_vmcnt<2 * LOADS>();
        else if (behind >= 1) wait_vmcnt<LOADS>();
        else wait_vmcnt<0>();
        work(x);
      }
    }
    // the wavefronts' sums, through LDS
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] += __shfl_xor(l[nt], 16, 64);
      l[nt] += __shfl_xor(l[nt], 32, 64);
#pragma unroll
      for (int d = 0; d < TILES; ++d)  // (what is right of a column)
        if (PARTS == 1 || part == d / 2 / OWN) *(f32x4*)((float*)ring[wave] + (R * nt + r16) * OUT_P + 16 * d + 4 * qd) = acc[nt][d];
      if (qd == 0 && part == 0) { stats[0][wave][R * nt + r16] = top[nt] * P.scale_log2e; stats[1][wave][R * nt + r16] = l[nt]; }
    }
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
        x += f * *(const f32x4*)((const float*)ring[w] + r * OUT_P + 4 * c);
      }
      const int j = token(m0 + r), hh = g * P.G + m0 + r - j * P.G;
      const int64_t row = (int64_t)(t.row0 + j) * P.Hq + hh;
      const float inv = sum == 0.f ? 0.f : 1.0f / sum, lse2 = sum == 0.f ? -__builtin_inff() : best + __builtin_log2f(sum);  // (a sum that is no number is passed on)
      x *= inv;
      if (whole) {
        store4((T*)P.o + row * D + 4 * c, x);
        if (c == 0) P.lse[(int64_t)hh * P.T + t.row0 + j] = lse2 * 0.69314718055994531f;
      } else {  // place 0: an item that began before this workgroup's strips, 1: one that ends behind them
        const int64_t at = ((int64_t)blockIdx.x * 2 + (x_first == item.first)) * ROWS + r;
        if (c == 0) P.part_lse[at] = lse2;
        *(f32x4*)(P.part_o + at * D + 4 * c) = x;
      }
    }
    if (!whole && x_first == item.first) cut = CutItem{t.row0, rows, m0, g, parts_of(item.first + item.count - 1, share), {}};
    x_first = x_next;
    if (x_first >= x_end) break;
    __syncthreads();  // the sums' LDS is free
    item = stream.find(A, x_first, lane, false);  // (loaded again: kept, the sequences' numbers would cost the strips registers)
  }
  if (P.splits != 1 && threadIdx.x == 0) A.cuts[blockIdx.x] = cut;  // every workgroup, so that nothing of an earlier call is left
}

// Joins the parts of the items that were cut: a workgroup to some rows of an item that began in workgroup blockIdx.x of the launch before, each of its NG groups of threads every NG-th part, RUNS
// of them on their way at a time.  Few rows have many parts, so there are as many groups as there is room for beside four rows.  Chunks have two or three, and many rows, so one group takes
// all of them (2 x 2000 tokens, 67 MB of parts: 48 us by four groups of 8 parts, 14 so).  A part that saw nothing has LSE -infinity; one that saw what is no number has left that, and so is
// the row's result.
constexpr int join_groups(int D, int rows) { return rows <= 32 ? 512 / D : 1; }
constexpr int join_rows(int D, int rows) { return 4 * 512 / D / join_groups(D, rows); }  // of a workgroup
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(512) void cache4_join_kernel(Cache4Params A) {
  const WindowParams& P = A.w;
  constexpr int NG = join_groups(D, ROWS), RUNS = NG > 1 ? 8 : 2, MINE = join_rows(D, ROWS), LANES = D / 4;
  const CutItem cut = A.cuts[blockIdx.x];
  const int group = threadIdx.x / (MINE * LANES), lane = threadIdx.x % (MINE * LANES), r = lane / LANES, c = 4 * (lane % LANES);
  const int m = cut.m0 + MINE * (int)blockIdx.y + r;
  if (cut.parts == 0 || m - r >= cut.rows) return;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  float best = -__builtin_inff(), sum = 0.f;
  for (int z0 = group; z0 < cut.parts; z0 += NG * RUNS) {
    float lse[RUNS], top = best;
    f32x4 part[RUNS];
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {  // (past the last part, it again)
      const int z = min(z0 + NG * i, cut.parts - 1);
      const int64_t from = (((int64_t)blockIdx.x + z) * 2 + (z == 0)) * ROWS + MINE * blockIdx.y + r;
      lse[i] = P.part_lse[from];
      part[i] = *(const f32x4*)(P.part_o + from * D + c);
      if (z0 + NG * i >= cut.parts) lse[i] = -__builtin_inff();
    }
#pragma unroll
    for (int i = 0; i < RUNS; ++i) top = fmaxf(top, lse[i]);
    const float ref = top == -__builtin_inff() ? 0.f : top;  // nothing seen yet: keep the exponents finite
    const float old = fast_exp2(best - ref);
    sum *= old;
    x *= old;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const float f = fast_exp2(lse[i] - ref);
      sum += f;
      if (lse[i] != -__builtin_inff()) x += f * part[i];
    }
    best = top;
  }
  if constexpr (NG > 1) {
    __shared__ __attribute__((aligned(16))) float sums[NG][MINE][D + 4];  // (and what they are relative to, their weight)
    *(f32x4*)&sums[group][r][c] = x;
    if (c == 0) { sums[group][r][D] = best; sums[group][r][D + 1] = sum; }
    __syncthreads();
    if (group > 0) return;
    best = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < NG; ++w) best = fmaxf(best, sums[w][r][D]);
    sum = 0.f;
    x = f32x4{0.f, 0.f, 0.f, 0.f};
    const float ref = best == -__builtin_inff() ? 0.f : best;
#pragma unroll
    for (int w = 0; w < NG; ++w) {
      const float f = fast_exp2(sums[w][r][D] - ref);
      sum += f * sums[w][r][D + 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(f, sums[w][r][c + e], x[e]);
    }
  }
  if (m >= cut.rows) return;
  const int j = (int)((unsigned)m / (unsigned)P.G), h = cut.g * P.G + m - j * P.G, tok = cut.row0 + j;
  x *= sum == 0.f ? 0.f : 1.0f / sum;
  store4((T*)P.o + ((int64_t)tok * P.Hq + h) * D + c, x);
  if (c == 0) P.lse[(int64_t)h * P.T + tok] = sum == 0.f ? -__builtin_inff() : (best + __builtin_log2f(sum)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------------------
// Many rows (bfloat16): the forward of packed batches (window_fwd_rows) over tiles that are expanded on their way into LDS.  Every value held is a bfloat16 number, so nothing is rounded on
// the way.  Eight wavefronts of 32 rows share a tile: its expansion, two vector instructions an element, is then a third of what the products and probabilities of the tile take.
// Wavefronts 0 .. 3 expand 16 rows of K each, a lane a quarter of a row (eight elements of every group of 32); wavefronts 4 .. 7 those of V, a lane four words of a row.  Codes of the
// tile after the next are on their way to registers while the next one is expanded and the present one multiplied.
constexpr int kChunkWaves = 8;
template <int D>
struct ExpandedTiles {
  static constexpr int GROUPS = D / 32, TILE_B = 64 * D * 2;
  unsigned long long codes;  // of page 0, this KV head
  unsigned long long steps;
  unsigned code[GROUPS], step[GROUPS / 2];
  unsigned at;     // where the lane's elements go in a tile
  int row, part;   // of the tile; of the row
  bool value;
  PagesAhead<D> ahead;
  __device__ inline void init(const Cache4Params& A, const RowTile& t, const KeySource<D, true>& src, int g, int wave, int lane, unsigned tiles0) {
    value = wave >= 4;
    codes = (unsigned long long)(value ? A.cache.v : A.cache.k) + ((unsigned long long)g << A.cache.page_shift) * (D / 2);
    steps = (unsigned long long)(value ? A.cache.v_step : A.cache.k_step) + ((unsigned long long)g << A.cache.page_shift) * (GROUPS * 2);
    row = 16 * (wave & 3) + (lane >> 2);
    part = lane & 3;
    at = tiles0 + (value ? TILE_B : 0) + row * (D * 2);
  }
  __device__ __attribute__((always_inline)) inline int first_row(const KeyTiles<64>& keys, int x) const { return 64 * keys.at(x) + __builtin_amdgcn_readfirstlane(row & ~15); }
  __device__ __attribute__((always_inline)) inline void look_up(const Cache4Params& A, const KeyTiles<64>& keys, const KeySource<D, true>& src, int x, int count) {
    ahead.look_up(A.w, src, first_row(keys, min(x, count - 1)));
  }
  __device__ __attribute__((always_inline)) inline void look_up_all(const Cache4Params& A, const KeyTiles<64>& keys, const KeySource<D, true>& src, int x, int count) {
    ahead.look_up_all(A.w, src, 64 * keys.at(min(x, count - 1)), part);
  }
  __device__ __attribute__((always_inline)) inline unsigned missing(const Cache4Params& A, const KeyTiles<64>& keys, const KeySource<D, true>& src, int x) const {
    return ahead.missing(A.w, src, 64 * keys.at(x), part);
  }
  // codes of tile x (its page is known); rows that are not there are zeros
  __device__ __attribute__((always_inline)) inline void load(const Cache4Params& A, const KeyTiles<64>& keys, const KeySource<D, true>& src, int x) {
    int there;
    const unsigned long long from = ahead.rows_at(A.w, src, first_row(keys, x), there);
    const unsigned rows = __builtin_amdgcn_readfirstlane(there);
    auto scalar = [](unsigned long long a) __attribute__((always_inline)) {  // (else a loop over the lanes' resources, which are all the same)
      return (const void*)(((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)a));
    };
    const Rsrc rc = resource(scalar(codes + from * (D / 2)), rows * (D / 2)), rs = resource(scalar(steps + from * (GROUPS * 2)), rows * GROUPS * 2);
    const int r = row & 15;
    if constexpr (D == 128) {
      const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(rc, r * (D / 2) + part * (D / 8), 0, 0);
      const u32x2 z = __builtin_amdgcn_raw_buffer_load_b64(rs, r * GROUPS * 2, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) code[e] = y[e];
      step[0] = z[0]; step[1] = z[1];
    } else {
      const u32x2 y = __builtin_amdgcn_raw_buffer_load_b64(rc, r * (D / 2) + part * (D / 8), 0, 0);
      code[0] = y[0]; code[1] = y[1];
      step[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, r * GROUPS * 2, 0, 0);
    }
  }
  __device__ __attribute__((always_inline)) inline void expand(int buffer) const {
    const unsigned to = at + buffer * 2 * TILE_B;
    const int swizzle = chunk_swizzle<D>(row);
    if (!value) {  // word c: elements 32 c + 8 part + (0 .. 7)
#pragma unroll
      for (int c = 0; c < GROUPS; ++c) {
        const float f = step_at(step[c / 2], c);
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x2 z = e == 0 ? numbers<0>(code[c]) : e == 1 ? numbers<1>(code[c]) : e == 2 ? numbers<2>(code[c]) : numbers<3>(code[c]);
          y[2 * e] = (bf16)(z[0] * f);
          y[2 * e + 1] = (bf16)(z[1] * f);
        }
        *(bf16x8 __attribute__((address_space(3)))*)(uintptr_t)(to + 16 * ((4 * c + part) ^ swizzle)) = y;
      }
    } else {  // words i = 4 part + (0 .. 3) of D/8 bits: byte e of word i holds elements 32 e + i and 32 e + 16 + i
#pragma unroll
      for (int e = 0; e < GROUPS; ++e) {
        const float f = step_at(step[e / 2], e);
        bf16x4 lo, hi;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          f32x2 z;
          if constexpr (D == 128) z = e == 0 ? numbers<0>(code[w]) : e == 1 ? numbers<1>(code[w]) : e == 2 ? numbers<2>(code[w]) : numbers<3>(code[w]);
          else z = 2 * (w & 1) + e == 0 ? numbers<0>(code[w / 2]) : 2 * (w & 1) + e == 1 ? numbers<1>(code[w / 2]) : 2 * (w & 1) + e == 2 ? numbers<2>(code[w / 2]) : numbers<3>(code[w / 2]);
          lo[w] = (bf16)(z[0] * f);
          hi[w] = (bf16)(z[1] * f);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int d = 32 * e + 16 * half;  // and 4 part
          *(bf16x4 __attribute__((address_space(3)))*)(uintptr_t)(to + 16 * (((d >> 3) + (part >> 1)) ^ swizzle) + 8 * (part & 1)) = half ? hi : lo;
        }
      }
    }
  }
  __device__ __attribute__((always_inline)) inline void start(const Cache4Params& A, const KeyTiles<64>& keys, const KeySource<D, true>& src, int begin, int count) {
    if (begin >= count) return;
    look_up(A, keys, src, begin, count);
    look_up_all(A, keys, src, begin, count);
    load(A, keys, src, begin);
    look_up(A, keys, src, begin + 1, count);
    expand(0);
    if (begin + 1 < count) load(A, keys, src, begin + 1);
    look_up(A, keys, src, begin + 2, count);
  }
  __device__ __attribute__((always_inline)) inline void arrive(const Cache4Params& A, const KeyTiles<64>& keys, const KeySource<D, true>& src, int x, int begin, int count) {
    __syncthreads();
    if (x + 1 < count) expand((x + 1 - begin) & 1);
    if (x + 2 < count) load(A, keys, src, x + 2);
    look_up(A, keys, src, x + 3, count);
    look_up_all(A, keys, src, x + 1, count);
  }
};
// An item a workgroup, the last tiles of rows of a sequence first; its keys in P.splits runs, joined by cache_merge_kernel.
template <int D>
__global__ __launch_bounds__(64 * kChunkWaves) __attribute__((amdgpu_waves_per_eu(2))) void cache4_chunk_kernel(Cache4Params A) {
  __shared__ __attribute__((aligned(1024))) char tiles[2][2][64 * D * 2];  // [buffer][K, V]
  const WindowParams& P = A.w;
  const int z = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (unsigned)P.Hkv % (unsigned)P.splits));
  const RowTile t = locate_tile<32 * kChunkWaves, true>(P, blockIdx.x / (unsigned)P.Hkv / (unsigned)P.splits);
  if (t.s < 0) return;
  const int g = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % (unsigned)P.Hkv));
  const int64_t from = (int64_t)z * P.per_split, to = z < P.splits - 1 ? from + P.per_split : 0x7fffffff;
  window_fwd_rows<D, true, kChunkWaves, ExpandedTiles<D>>(P, &tiles[0][0][0], A, t, g, threadIdx.x & 63, from, to, P.splits > 1,
                                                          [&](int i, int h, int) __attribute__((always_inline)) { return ((int64_t)z * P.T + t.row0 + i) * P.Hq + h; });
}
// Equal shares of the stream of 64-key tiles.  (A kernel of its own: the loop over items costs a workgroup of one item 4 %.)
template <int D>
__global__ __launch_bounds__(64 * kChunkWaves) __attribute__((amdgpu_waves_per_eu(2))) void cache4_chunk_stream_kernel(Cache4Params A) {
  constexpr int ROWS = 32 * kChunkWaves;
  __shared__ __attribute__((aligned(1024))) char tiles[2][2][64 * D * 2];  // [buffer][K, V]
  const int lane = threadIdx.x & 63;
  Stream<ROWS, 64> stream;
  const int share = stream.share(A, gridDim.x, 8, lane);
  const int64_t x_last = (int64_t)share * (blockIdx.x + 1);
  int x_first = (int)min(x_last - share, (int64_t)0x7fffffff);  // (the stream ends before)
  const int x_end = (int)min(x_last, (int64_t)0x7fffffff);
  Item item = stream.find(A, x_first, lane, true);
  CutItem cut{};
  while (item.t.s >= 0) {
    const int x_next = min(x_end, item.first + item.count);
    const bool begins = x_first == item.first, part = !begins || x_next != item.first + item.count;
    const int64_t at = ((int64_t)blockIdx.x * 2 + begins) * ROWS;
    int here = lane;
    asm volatile("" : "+v"(here));  // (what follows from it stays in the loop: in front of it, it would be kept, and spilled)
    window_fwd_rows<D, true, kChunkWaves, ExpandedTiles<D>>(A.w, &tiles[0][0][0], A, item.t, item.g, here, (int64_t)(x_first - item.first) << A.unit,
                                                            part ? (int64_t)(x_next - item.first) << A.unit : 0x7fffffff, part,
                                                            [&](int, int, int row) __attribute__((always_inline)) { return at + row; });
    if (part && begins) cut = CutItem{item.t.row0, item.t.n * A.w.G, item.t.tile * ROWS, item.g, parts_of(item.first + item.count - 1, share), {}};
    x_first = x_next;
    if (x_first >= x_end) break;
    __syncthreads();  // the tiles' LDS is free
    item = stream.find(A, x_first, lane, false);
  }
  if (threadIdx.x == 0) A.cuts[blockIdx.x] = cut;
}

// How the work is cut.  Sequences of up to kFewRows4 flattened rows are cache4_split_kernel's (float32: all of them), the others cache4_chunk_kernel's; a batch of one kind costs one launch.
// 8 sequences of 20000 tokens, 32/8 heads, with 32, 64, 96 and 128 rows: 72, 113, 150 and 190 us by the first, 146, 150, 153 and 160 by the second.
constexpr int kFewRows4 = 64;
struct Cache4Plan {
  int64_t few, many;      // tiles of rows; 0: no such launch
  int rows;               // of a tile of few rows
  int workgroups;         // of few rows; 0: whole items, a workgroup each
  int unit;
  int many_workgroups;    // of many rows, in equal shares; 0: whole items, their keys in `splits` runs of per_split tiles
  int splits, per_split;
  size_t part_lse, part_o, bytes;
};
static Cache4Plan plan_cache4(const sb_cache4* c, const sb_chunk* n, int window, int sinks) {
  Cache4Plan p{};
  const int G = n->num_q_heads / c->num_kv_heads, S = n->num_seqs, D = c->head_dim;
  const bool f32 = c->dtype == SB_F32;
  const int64_t most = (int64_t)std::min(n->max_new, n->total_new) * G;  // rows of a sequence
  auto items = [&](int64_t most_rows, int rows) { return std::min(row_tiles_most(n->total_new, S, G, rows), (most_rows + rows - 1) / rows * S); };
  auto tiles = [&](int rows, int tile) {  // of keys of an item, about: what max_length, the page table, the window and the sinks leave
    const int64_t in_window = (int64_t)window + (rows + G - 1) / G + sinks + 2 * tile;
    const int64_t longest = std::min<int64_t>(n->max_length, (int64_t)c->max_pages * c->page_size);
    return (std::min(in_window, longest) + tile - 1) / tile;
  };
  // (32 rows a tile cost 1.55 to 1.9 times what 16 do: two tiles' worth where their number is even, three in two would not pay.  8 sequences of 20000, 32/8 heads, 64 rows: 144 us in tiles of 16, 113 of 32;
  // 64 of 500 to 8000, 28/4 heads, 35 rows: 96 us in tiles of 16, 99 of 32.  Float32, where a row's numbers take three times the registers, in tiles of 16 and 32: 16 of 500 to 20000, 32/8 heads, 32 rows 74
  // and 114, 64 rows 131 and 192;  16/4 heads of 64, 32 rows 32 and 40;  2000 behind 20000 2690 and 4340, a prompt of 2000 195 and 304.)
  auto unit_of = [&](int64_t items, int tile) {  // see Stream
    const int64_t strips = ((int64_t)c->max_pages * c->page_size + tile - 1) / tile + 2;  // of an item, at most
    int unit = 0;
    while (items * (((strips - 1) >> unit) + 1) > 0x40000000ll && unit < 26) ++unit;
    return unit;
  };
  p.rows = most <= 4 && D == 128 ? 4 : most <= 8 ? 8 : f32 || (most + 15) / 16 % 2 != 0 ? 16 : 32;
  if (f32) p.few = items(most, p.rows);
  else if (G <= kFewRows4 && (S > 1 || most <= kFewRows4)) p.few = items(std::min<int64_t>(most, kFewRows4), p.rows);
  size_t sums = 0;
  if (p.few > 0) {
    // Whole items, without the launch that joins parts, where a wavefront has few strips of an item, or not many and there are many items; and for float32 prompts, whose items are many and
    // alike.  Else equal shares, for as many workgroups as the chip holds, or as have a strip a wavefront if sequences are as long as they may be: one long sequence among short ones would be
    // waited for.
    //   32/8 heads, equal shares and whole items, in us: one sequence of 400 14.9 and 10.8, of 1000 12.8 and 13.7, of 2000 14.9 and 21.1;  16 of 1000 19.3 and 14.0, of 2000 22.7 and 22.3;  64 of
    //   2000 39.8 and 30.9, of 100 to 2000 32.1 and 23.9, four of 2000 and 60 of 200 21.4 and 22.3;  64 of 4000 61.9 and 53.8, of 500 to 4000 39.2 and 41.0, one of 4000 and 63 of 100 16 and 37
    //   float32 chunks, likewise (items in brackets): 300 behind 8000 193 and 222 (600), 512 307 and 294 (1024), 700 441 and 428 (1400), 1200 778 and 717 (2400);  2 x 600 behind 1000 to 8000, 14/2 heads of
    //   64 183 and 196 (1052), 2 x 800 242 and 234 (1400);  2 x 800, 28/4 heads 838 and 745 (2800);  16 x 50, one of them behind 20000, the others 100 190 and 238 (1408), 8 x 100 288 and 239 (1408);
    //   2000 behind 20000 3060 and 2690 (4000);  a prompt of 6001 2470 and 1285 (12008)
    const int64_t of_wave = (tiles(p.rows, 32) + kWaves4 - 1) / kWaves4, all = p.few * c->num_kv_heads;
    if (!(of_wave <= 8 || (of_wave <= 16 && all >= 256) || (f32 && most > kFewRows4 && all >= 1280)))
      p.workgroups = (int)std::min<int64_t>(256 * split_waves(D, p.rows, f32 ? 3 : 1), all * of_wave);
    sums = (size_t)p.workgroups * 2 * p.rows;
    p.unit = unit_of(p.few * c->num_kv_heads, 32);
  }
  if (!f32 && most > kFewRows4) {
    p.many = items(most, 32 * kChunkWaves);
    // Very few items: their keys in runs of 8 tiles or more.  Else equal shares where the keys are mostly cached or behind a window, so that items are alike, and whole ones would not fill the
    // chip evenly.  The others, a first prompt's, are of all lengths, the longest first, and even out by themselves.
    //   runs, whole items and shares, in us: one chunk of 200 behind 30000, 32/8 heads 148, 910, 154;  1000 behind 8000, one head 33, 275, 41;  two of 2000 behind 20000 and 30000,
    //   window 8192, 28/4 heads (440 items) -, 539, 483;  three of 700 behind 5000 to 20000 1021, 636, 415;  a prompt of 6001 -, 342, 587, of 1000 76, 40, 75;  of 2000, 4/2 heads 46, 67, 59
    const int64_t workgroups = p.many * c->num_kv_heads, rounds = (workgroups + 255) / 256, all = tiles(32 * kChunkWaves, 64);
    p.splits = 1;
    if (workgroups < 64) {
      p.per_split = (int)std::max<int64_t>(((all * workgroups + 255) / 256 + 7) / 8 * 8, 8);
      p.splits = (int)std::max<int64_t>((all + p.per_split - 1) / p.per_split, 1);
      if (p.splits > 1) sums = std::max(sums, (size_t)p.splits * n->total_new * n->num_q_heads);
    } else if (64 * all >= 4 * (int64_t)n->max_new && workgroups < 2048 && (8 * rounds * 256 > 9 * workgroups || (S > 1 && workgroups < 1024))) {
      p.many_workgroups = 256;
      p.splits = 0;
      sums = std::max(sums, (size_t)p.many_workgroups * 2 * 32 * kChunkWaves);
      p.unit = std::max(p.unit, unit_of(workgroups, 64));
    }
  }
  p.part_lse = align_up(std::max(p.workgroups, p.many_workgroups) * sizeof(CutItem));
  p.part_o = align_up(p.part_lse + sums * sizeof(float));
  p.bytes = align_up(p.part_o + sums * D * sizeof(float));
  return p;
}
static int check_cache4_attn(const sb_cache4* c, const sb_chunk* n, int32_t window, int32_t sinks) {
  const int rc = check_cache4(c, n);
  if (rc != SB_OK) return rc;
  if (window < 1 || sinks < 0) { set_error("window (%d) must be at least 1 and sinks (%d) not negative", window, sinks); return SB_ERR_INVALID_ARG; }
  return check_rows(n->total_new, n->num_q_heads / c->num_kv_heads);
}

}  // namespace sb

using namespace sb;

extern "C" {

int sb_cache4_attn_ws_bytes(const sb_cache4* c, const sb_chunk* n, int32_t window, int32_t sinks, int64_t* bytes) {
  if (!bytes) { set_error("null output"); return SB_ERR_INVALID_ARG; }
  const int rc = check_cache4_attn(c, n, window, sinks);
  if (rc != SB_OK) return rc;
  *bytes = n->num_seqs == 0 || n->max_new == 0 ? 0 : (int64_t)plan_cache4(c, n, window, sinks).bytes;
  return SB_OK;
}

int sb_cache4_attn(const sb_cache4* c, const sb_chunk* n, int32_t window, int32_t sinks, const void* q, void* o, float* lse, void* ws, void* stream) {
  int rc = check_cache4_attn(c, n, window, sinks);
  if (rc != SB_OK) return rc;
  if (n->total_new == 0 || n->num_seqs == 0 || n->max_new == 0) return SB_OK;
  if (!q || !o || !lse) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if ((rc = check_cache4_arrays(c, n)) != SB_OK) return rc;
  const void* const buffers[] = {q, o, c->k, c->v, c->k_step, c->v_step, ws};
  if ((rc = check_aligned(buffers, 7)) != SB_OK) return rc;
  Cache4Params A{};
  WindowParams& P = A.w;
  P.q = q; P.o = o; P.lse = lse; P.cu = n->cu_new; P.cached = n->cached; P.max_new = n->max_new;
  P.T = n->total_new; P.S = n->num_seqs; P.Hq = n->num_q_heads; P.Hkv = c->num_kv_heads; P.G = P.Hq / P.Hkv;
  P.window = window; P.sinks = sinks;
  P.scale = n->softmax_scale > 0.f ? n->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
  P.scale_log2e = P.scale * 1.4426950408889634f;
  A.cache = make_paged(c);
  P.cache = PagedCache{nullptr, nullptr, c->page_table, c->num_pages, c->max_pages, c->page_size, A.cache.page_shift, c->num_kv_heads};
  const Cache4Plan plan = plan_cache4(c, n, window, sinks);
  if (plan.workgroups > 0 || plan.many_workgroups > 0 || plan.splits > 1) {
    if (!ws) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
    A.cuts = (CutItem*)ws;
    P.part_lse = (float*)((char*)ws + plan.part_lse);
    P.part_o = (float*)((char*)ws + plan.part_o);
  }
  const bool f32 = c->dtype == SB_F32;
  A.unit = plan.unit;
  if ((plan.few + plan.many) * P.Hkv > 0x40000000ll) { set_error("too many tiles for one launch"); return SB_ERR_UNSUPPORTED; }
  dim3 few_grid, many_grid, all_rows;
  if ((rc = grid_of(plan.workgroups > 0 ? plan.workgroups : plan.few * P.Hkv, 64 * kWaves4, &few_grid)) != SB_OK ||
      (rc = grid_of(plan.many_workgroups > 0 ? plan.many_workgroups : plan.many * P.Hkv * plan.splits, 64 * kChunkWaves, &many_grid)) != SB_OK ||
      (plan.splits > 1 && (rc = grid_of((int64_t)P.T * P.Hq, 256, &all_rows)) != SB_OK))
    return rc;
  const hipStream_t st = (hipStream_t)stream;
  KernelTimer kt(K_CACHE_ATTN, st);
  if (plan.many > 0) {
    P.splits = plan.splits; P.per_split = plan.per_split; P.part_rows = P.T;
    P.rows_from = plan.few > 0 ? kFewRows4 + 1 : 0;
    P.rows_to = 0x7fffffff;
    auto launch = [&](auto d) {
      constexpr int DD = decltype(d)::value;
      if (plan.many_workgroups > 0) {
        hipLaunchKernelGGL((cache4_chunk_stream_kernel<DD>), many_grid, dim3(64 * kChunkWaves), 0, st, A);
        SB_LAUNCH_CHECK("cache4_chunk_stream_kernel");
        hipLaunchKernelGGL((cache4_join_kernel<bf16, DD, 32 * kChunkWaves>), dim3(plan.many_workgroups, 32 * kChunkWaves / join_rows(DD, 32 * kChunkWaves)), dim3(512), 0, st, A);
        SB_LAUNCH_CHECK("cache4_join_kernel");
        return (int)SB_OK;
      }
      hipLaunchKernelGGL((cache4_chunk_kernel<DD>), many_grid, dim3(64 * kChunkWaves), 0, st, A);
      SB_LAUNCH_CHECK("cache4_chunk_kernel");
      return P.splits > 1 ? launch_cache_merge(P, DD, SB_BF16, all_rows, 0, st) : (int)SB_OK;
    };
    if ((rc = c->head_dim == 128 ? launch(std::integral_constant<int, 128>()) : launch(std::integral_constant<int, 64>())) != SB_OK) return rc;
  }
  if (plan.few > 0) {
    P.splits = plan.workgroups > 0 ? 0 : 1;
    P.rows_from = 0;
    P.rows_to = f32 ? 0x7fffffff : kFewRows4;
    auto launch = [&](auto ty, auto d, auto rows, auto pieces) {
      typedef decltype(ty) Type;
      constexpr int DD = decltype(d)::value, ROWS = decltype(rows)::value;
      hipLaunchKernelGGL((cache4_split_kernel<Type, DD, ROWS < 16 ? 16 / ROWS : 1, ROWS < 16 ? 1 : ROWS / 16, decltype(pieces)::value>), few_grid, dim3(64 * kWaves4), 0, st, A);
      SB_LAUNCH_CHECK("cache4_split_kernel");
      if (plan.workgroups > 0) {
        hipLaunchKernelGGL((cache4_join_kernel<Type, DD, ROWS>), dim3(plan.workgroups, ROWS / join_rows(DD, ROWS)), dim3(512), 0, st, A);
        SB_LAUNCH_CHECK("cache4_join_kernel");
      }
      return (int)SB_OK;
    };
    auto with_rows = [&](auto ty, auto d, auto pieces) {
      if constexpr (decltype(d)::value == 128)
        if (plan.rows == 4) return launch(ty, d, std::integral_constant<int, 4>(), pieces);
      if (plan.rows == 8) return launch(ty, d, std::integral_constant<int, 8>(), pieces);
      if constexpr (decltype(pieces)::value == 1)
        if (plan.rows == 32) return launch(ty, d, std::integral_constant<int, 32>(), pieces);
      return launch(ty, d, std::integral_constant<int, 16>(), pieces);
    };
    auto with_d = [&](auto ty, auto pieces) {
      return c->head_dim == 128 ? with_rows(ty, std::integral_constant<int, 128>(), pieces) : with_rows(ty, std::integral_constant<int, 64>(), pieces);
    };
    return f32 ? with_d(float(), std::integral_constant<int, 3>()) : with_d(bf16(), std::integral_constant<int, 1>());
  }
  return SB_OK;
}

}  // extern "C"
