// The paged cache in four bits: what its kernels share.
//
// 32 neighbouring elements of a head share a step; an element is the step times one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign (the chip's four-bit floating-point format).  A step has six
// significant bits and a level two, so every value held is a bfloat16 number.  Bytes of a row lie as the matrix instructions take them, so that a lane's operands of all groups of
// 32 are one load: keys in four pieces, piece b with elements 32 c + 8 b + (0 .. 7) of every group c; values in 16 words, word i with elements 16 j + i.
#pragma once

#include "sb_cache.h"

namespace sb {

struct PagedCache4 {
  unsigned char *k, *v;
  bf16 *k_step, *v_step;
  const int32_t* table;
  int num_pages, max_pages, page_size, page_shift, Hkv;
  // Row of token `pos` of sequence s and KV head g, or -1: no page.
  __device__ inline int64_t row_of(int s, int64_t pos, int g) const {
    const int64_t j = pos >> page_shift;
    if (j < 0 || j >= max_pages) return -1;
    const int page = table[(int64_t)s * max_pages + j];
    if (page < 0 || page >= num_pages) return -1;
    return (((int64_t)page * Hkv + g) << page_shift) + (pos & (page_size - 1));
  }
};

int check_cache4(const sb_cache4* c, const sb_chunk* n);
int check_cache4_arrays(const sb_cache4* c, const sb_chunk* n);
PagedCache4 make_paged(const sb_cache4* c);

}  // namespace sb
