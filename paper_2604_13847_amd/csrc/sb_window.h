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
  float* delta;       // [Hq][T] rowsum(dO * O), backward
  void *dq, *dk, *dv;
  const int32_t* cu;  // [S+1]: packed rows of the sequences (paged: of their new tokens)
  int T, S, Hq, Hkv, G;
  int window, sinks;
  float scale, scale_log2e;
  // a chunk over a paged cache
  PagedCache cache;
  const int32_t* cached;
  int max_new;
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
    int row0 = 0, n = 0;
    if (base + lane < P.S) {
      row0 = P.cu[base + lane];
      n = P.cu[base + lane + 1];
      if (PAGED) {
        row0 = min(max(row0, 0), P.T);
        n = min(n, P.T);
      }
      n = max(n - row0, 0);
      if (PAGED) n = min(n, P.max_new);
    }
    const int64_t c = ((int64_t)n * P.G + ROWS - 1) / ROWS;
    int64_t incl = c;
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t t = __shfl_up(incl, off, 64);
      if (lane >= off) incl += t;
    }
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(x < incl);
    const int src = hit ? __builtin_ctzll(hit) : 63;
    if (hit) {
      RowTile t;
      t.s = base + src;
      t.row0 = __builtin_amdgcn_readlane(row0, src);
      t.n = __builtin_amdgcn_readlane(n, src);
      const int64_t first = __shfl(incl - c, src, 64), tiles = __shfl(c, src, 64);
      t.tile = __builtin_amdgcn_readfirstlane((int)(tiles - 1 - (x - first)));
      t.pos0 = PAGED ? min(max(P.cached[t.s], 0), 0x7fffffff - t.n) : 0;
      return t;
    }
    x -= __shfl(incl, 63, 64);
  }
  return RowTile{-1, 0, 0, 0, 0};
}

// Keys of rows at positions ta .. tb, in tiles of `TILE`: sink tiles 0 .. far - 1, then tiles near .. end - 1.  (tb: that of the last key that can exist, if that is less.)
template <int TILE>
struct KeyTiles {
  int far, near, end;
  __device__ inline KeyTiles(int ta, int tb, int window, int sinks) {
    near = max(0, ta - window + 1) / TILE;
    end = max(tb / TILE + 1, near);
    far = min((int)(((int64_t)sinks + TILE - 1) / TILE), near);
  }
  __device__ inline int count() const { return far + end - near; }
  __device__ inline int at(int i) const { return i < far ? i : near + i - far; }
};
__device__ inline bool sees(int t, int u, int window, int sinks) { return u <= t && (t - u < window || u < sinks); }

int64_t row_tiles(const int32_t* cu_host, int S, int G, int rows);  // of a packed batch
int64_t row_tiles_most(int total, int S, int G, int rows);          // where the lengths are not known to the host

// Forward launch of all query rows; P is complete.  dtype as in sb_problem.
int launch_window_fwd(const WindowParams& P, int D, int dtype, bool paged, int64_t tiles32, int64_t tiles, hipStream_t st);

}  // namespace sb
