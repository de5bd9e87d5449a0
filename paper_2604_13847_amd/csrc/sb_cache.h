// What the kernels see of a paged cache, and where a packed row belongs.
#pragma once

#include "sb_internal.h"

namespace sb {

struct PagedCache {
  void *k, *v;
  const int32_t* table;
  int num_pages, max_pages, page_size, page_shift, Hkv;
  // Row (of head_dim elements) of token `pos` of sequence s and KV head g in k and v, or -1: no page.
  __device__ inline int64_t row_of(int s, int64_t pos, int g) const {
    const int64_t j = pos >> page_shift;
    if (j < 0 || j >= max_pages) return -1;
    const int page = table[(int64_t)s * max_pages + j];
    if (page < 0 || page >= num_pages) return -1;
    return (((int64_t)page * Hkv + g) << page_shift) + (pos & (page_size - 1));
  }
};

// The sequence of packed row `tok`: the number of ends cu[s + 1] <= tok, S if there are no more.  All lanes of a wavefront call it; a step of 64 sequences is one load.
__device__ inline int sequence_of(const int32_t* cu, int S, int tok, int lane) {
  for (int base = 0; base < S; base += 64) {
    const bool behind = base + lane < S && cu[base + lane + 1] <= tok;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(behind));
    if (n < 64) return base + n;
  }
  return S;
}

int check_cache(const sb_cache* c, const sb_chunk* n);         // sizes and types
int check_cache_arrays(const sb_cache* c, const sb_chunk* n);  // addresses
PagedCache make_paged(const sb_cache* c);

}  // namespace sb
