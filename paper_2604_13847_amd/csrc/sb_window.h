// Shared by the kernels of window attention over packed batches and of a chunk's attention over a paged cache.
#pragma once

#include "sb_attn_common.h"
#include "sb_cache.h"

namespace sb {

struct WindowParams {
  const void *q, *k, *v, *d_o;
  const void* o_in;
  void* o;
  float* lse;         // [Hq][T]
  float* lse2;        // [T][Hq] LSE * log2 e and
  float* dr;          // rowsum(dO * O): backward, the order in which flattened rows need them (float32)
  bf16x8* stats;      // [T][Hq][2] the same as operands of matrix instructions (bfloat16), see split3
  float* partials;    // dK, dV of sinks from rows far behind, see window_dkv_kernel
  int far_rows;       // tokens of a far item
  float* parts;       // dK, dV of an item whose rows several workgroups share
  int near_parts;     // that many
  void *dq, *dk, *dv;
  const int32_t* cu;  // [S+1]: packed rows of the sequences (paged: of their new tokens)
  int T, S, Hq, Hkv, G;
  int window, sinks;
  float scale, scale_log2e;
  // a chunk over a paged cache
  PagedCache cache;
  const int32_t* cached;
  int max_new;
  // keys split over `splits` workgroups, per_split tiles each (the last one takes what is left); part_o [splits][part_rows][Hq][D] normalised, part_lse [splits][part_rows][Hq] in
  // base 2.  Row i of sequence s is there part_seq_rows * s + i or, where that is 0 (and part_rows T), the packed row.
  int splits, per_split;
  int part_rows, part_seq_rows;
  float *part_o, *part_lse;
  int rows_from, rows_to;  // sequences of these many flattened rows are this launch's, the others another's
};

// The query rows of a KV head's group are flattened: row m of a sequence is token m / G, query head m % G of the group.  Heads of a token so share
// the key tiles that they all need, whatever their number, and a single token's heads fill as much of a tile as they can.
struct RowTile {
  int s;          // sequence, or -1
  int tile;       // tile of it
  int row0, n;    // first packed row of the sequence, its rows
  int pos0;       // position of its first row
};

// Tile x of all sequences, each cut into tiles of ROWS flattened rows, a sequence's last tile first: it has the most keys.  All lanes of a wavefront call it; a
// step of 64 sequences costs a load and a scan.
template <int ROWS, bool PAGED>
__device__ inline RowTile locate_tile(const WindowParams& P, int64_t x) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < P.S; base += 64) {
    int row0 = 0, n = 0, pos0 = 0;
    if (base + lane < P.S) {
      row0 = P.cu[base + lane];
      n = P.cu[base + lane + 1];
      if (PAGED) {
        pos0 = max(P.cached[base + lane], 0);
        row0 = min(max(row0, 0), P.T);
        n = min(n, P.T);
      }
      n = max(n - row0, 0);
      if (PAGED) {
        n = min(n, P.max_new);
        if (n * P.G < P.rows_from || n * P.G > P.rows_to) n = 0;
        pos0 = min(pos0, 0x7fffffff - n);
      }
    }
    const int c = (int)(((unsigned)n * (unsigned)P.G + (unsigned)ROWS - 1) / (unsigned)ROWS);  // (rows of a sequence, and tiles of 64 of them, fit 31 bits: see check_rows)
    int incl = c;
    for (int off = 1; off < 64 && off < P.S - base; off <<= 1) {
      const int t = __shfl_up(incl, off, 64);
      if (lane >= off) incl += t;
    }
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(base + lane < P.S && x < incl);
    if (hit) {
      const int src = __builtin_ctzll(hit), tiles = __builtin_amdgcn_readlane(c, src);
      RowTile t;
      t.s = base + src;
      t.row0 = __builtin_amdgcn_readlane(row0, src);
      t.n = __builtin_amdgcn_readlane(n, src);
      t.pos0 = __builtin_amdgcn_readlane(pos0, src);
      t.tile = __builtin_amdgcn_readfirstlane(min(max(tiles - 1 - (int)(x - (__builtin_amdgcn_readlane(incl, src) - tiles)), 0), tiles - 1));
      return t;
    }
    x -= __builtin_amdgcn_readlane(incl, min(P.S - base, 64) - 1);
  }
  return RowTile{-1, 0, 0, 0, 0};
}

// x as three bfloat16 numbers that add up to it but for 2^-25 of it, followed by zeros: a product with (-1, -1, -1, 0, ...) subtracts x from an accumulator.
__device__ inline bf16x8 split3(float x) {
  bf16x8 r = zero_bf16x8();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    r[i] = (bf16)x;
    x -= (float)r[i];
  }
  return r;
}

// Keys of rows at positions ta .. tb, in tiles of `TILE`: sink tiles 0 .. far - 1, then tiles near .. end - 1.  (tb: that of the last key that can exist, if that is less; where all
// rows are behind it, there are sink tiles up to it and no others.)
template <int TILE>
struct KeyTiles {
  int far, near, end;
  __device__ inline KeyTiles(int ta, int tb, int window, int sinks) {
    near = max(0, ta - window + 1) / TILE;
    end = max(tb / TILE + 1, near);
    far = min((int)(((int64_t)sinks + TILE - 1) / TILE), min(near, tb / TILE + 1));
  }
  __device__ inline int count() const { return far + end - near; }
  __device__ inline int at(int i) const { return i < far ? i : near + i - far; }
};
__device__ inline bool sees(int t, int u, int window, int sinks) { return u <= t && (t - u < window || u < sinks); }
// the same question about key u0 + k + 4 hf of a tile at u0, k known at compile time: three comparisons with a constant
struct Sight {
  int t, w, s;
  __device__ inline Sight(int pos, int u0, int hf, int window, int sinks) : t(pos - u0 - 4 * hf), w(t - window), s(sinks - u0 - 4 * hf) {
    asm volatile("" : "+v"(t), "+v"(w), "+v"(s));  // (else the compiler keeps pos - k for every k in registers around the loop)
  }
  __device__ inline bool operator()(int k) const { return (k <= t) & ((k > w) | (k < s)); }
};

// One wavefront's part of copying a 64-key tile of K or V into LDS (layout as in sb_attn_common.h), NW wavefronts to a tile, as buffer loads whose resource covers
// the rows that exist, so that the others arrive as zeros.  A load's rows (4, or 8 at head_dim 64) lie in one page.
template <int D, int NW>
struct RowsLoader {
  static constexpr int MINE = 64 / NW, C = D / 8, RPI = 64 / C, LOADS = MINE / RPI;  // 16-byte chunks per row, rows per load, loads per wavefront
  unsigned voff[LOADS];
  unsigned pitch;  // bytes from row to row
  int wave;
  __device__ inline void init(unsigned pitch_, int wave_, int lane) {
    pitch = pitch_;
    wave = wave_;
#pragma unroll
    for (int a = 0; a < LOADS; ++a) {
      const int r = MINE * wave + a * RPI + lane / C;
      voff[a] = (lane / C) * pitch + 16 * ((lane % C) ^ chunk_swizzle<D>(r));
    }
  }
  // `rows` of the wavefront's rows exist, from `base` on (wave-uniform, by scalar instructions: see QuadLoader)
  __device__ inline void issue(unsigned long long base, int rows, unsigned slot) const {
#pragma unroll
    for (int a = 0; a < LOADS; ++a) {
      const int n = min(rows - a * RPI, RPI);
      const i32x4 rsrc = QuadLoader<D>::resource(base + (unsigned long long)(a * RPI) * pitch, n > 0 ? (unsigned)(n - 1) * pitch + D * 2 : 0u);
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" : : "v"(voff[a]), "s"(slot + (MINE * wave + a * RPI) * D * 2), "s"(rsrc) : "memory", "m0");
    }
  }
};

// Where the keys of a sequence and KV head lie, for wave-uniform questions.
template <int D, bool PAGED>
struct KeySource {
  unsigned long long k, v;  // first row (paged: of page 0)
  unsigned pitch;           // bytes from row to row
  const int32_t* pages;     // the sequence's row of the page table
  int end, lo;              // keys u with lo <= u < end or u < sinks are read
  __device__ inline void init(const WindowParams& P, const RowTile& t, int g, int lo_, int end_) {
    if (PAGED) {
      const unsigned long long o = ((unsigned long long)g << P.cache.page_shift) * (D * 2);
      k = (unsigned long long)P.cache.k + o;
      v = (unsigned long long)P.cache.v + o;
      pitch = D * 2;
      pages = P.cache.table + (int64_t)t.s * P.cache.max_pages;
    } else {
      const unsigned long long o = ((unsigned long long)t.row0 * P.Hkv + g) * (D * 2);
      k = (unsigned long long)P.k + o;
      v = (unsigned long long)P.v + o;
      pitch = (unsigned)P.Hkv * (D * 2);
      pages = nullptr;
    }
    end = end_;
    lo = lo_;
  }
  // rows u .. u + n - 1 of a packed batch: bytes from the first row, and how many exist from there on
  __device__ inline unsigned long long rows_at(const WindowParams& P, int u, int n, int& rows) const {
    rows = min(end - u, n);
    if (u + n <= lo && u >= P.sinks) rows = 0;
    return (unsigned long long)(unsigned)u * pitch;
  }
};

// Rows of a wavefront's 32, held as C tiles (lane%32: row, value(dt, v): column 32dt + c_row(v, lane/32)), to memory through LDS (`buf`, the wavefront's own, 32 rows), whole rows
// at a time; address(r): row r's, or null.  (store_rows in sb_attn_common.h, for rows that are no constant pitch apart.)
template <int D, typename V, typename A>
__device__ inline void store_tile(char* buf, int lane, V value, A address) {
  constexpr int C = D / 8, RPI = 64 / C;
  const int l32 = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int vg = 0; vg < 4; ++vg) {
      const int byte = (32 * dt + 8 * vg + 4 * hf) * 2;
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (bf16)value(dt, 4 * vg + e);
      *(bf16x4*)(buf + l32 * (D * 2) + 16 * ((byte >> 4) ^ (l32 & (C - 1))) + (byte & 15)) = y;
    }
  asm volatile("" ::: "memory");  // (LDS operations of a wavefront complete in order)
#pragma unroll
  for (int a = 0; a < 32 / RPI; ++a) {
    const int r = a * RPI + lane / C, c = lane % C;
    const f32x4 x = *(const f32x4*)(buf + r * (D * 2) + 16 * (c ^ (r & (C - 1))));
    bf16* to = address(r);
    if (to) *(f32x4*)(to + 8 * c) = x;
  }
}

int grid_of(int64_t workgroups, int threads, dim3* grid);  // a launch has fewer than 2^32 threads
int check_aligned(const void* const* p, int n);           // tensors are read and written 16 bytes at a time
int check_rows(int64_t tokens, int G);  // flattened rows fit 31 bits
constexpr int kSplitRows = 32;  // flattened rows of an item of cache_split_kernel
int64_t row_tiles(const int32_t* cu_host, int S, int G, int rows);  // of a packed batch
int64_t row_tiles_most(int total, int S, int G, int rows);          // where the lengths are not known to the host

// Forward launch of all query rows; P is complete.  dtype as in sb_problem; tiles: of forward_rows(dtype) flattened rows.
constexpr int kWaves = 4;  // of a forward or dQ workgroup (bfloat16)
constexpr int forward_rows(int dtype) { return dtype == SB_F32 ? 32 : 32 * kWaves; }
int launch_window_fwd(const WindowParams& P, int D, int dtype, bool paged, int64_t tiles, hipStream_t st);
// Joins the runs of keys that a launch before left in part_o and part_lse: a workgroup to a row and head, of all rows, or of the first seq_rows of every sequence.
int launch_cache_merge(const WindowParams& P, int D, int dtype, dim3 workgroups, int seq_rows, hipStream_t st);

}  // namespace sb
