// Attention of new tokens over a paged cache (serving).
#include <math.h>

#include "sb_window.h"

namespace sb {

int check_cache(const sb_cache* c, const sb_chunk* n) {
  if (!c || !n) { set_error("null cache or chunk"); return SB_ERR_INVALID_ARG; }
  if (c->dtype != SB_BF16 && c->dtype != SB_F32) { set_error("dtype must be SB_BF16 or SB_F32"); return SB_ERR_INVALID_ARG; }
  if (c->num_pages < 0 || c->max_pages < 0 || n->num_seqs < 0 || n->total_new < 0 || n->max_new < 0 || n->max_length < 0) {
    set_error("negative size");
    return SB_ERR_INVALID_ARG;
  }
  if (c->num_kv_heads < 1 || n->num_q_heads < 1 || n->num_q_heads % c->num_kv_heads != 0) {
    set_error("num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)", n->num_q_heads, c->num_kv_heads);
    return SB_ERR_INVALID_ARG;
  }
  if (c->head_dim != 64 && c->head_dim != 128) { set_error("head_dim %d unsupported (64 or 128)", c->head_dim); return SB_ERR_UNSUPPORTED; }
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0) {
    set_error("page_size %d unsupported (a power of two, 16 .. 1024)", c->page_size);
    return SB_ERR_UNSUPPORTED;
  }
  if ((int64_t)c->max_pages * c->page_size > 0x7fffffffll - 1024) { set_error("max_pages * page_size passes 32 bits"); return SB_ERR_UNSUPPORTED; }
  return SB_OK;
}
int check_cache_arrays(const sb_cache* c, const sb_chunk* n) {
  if (!n->cu_new || !n->cached) { set_error("cu_new and cached are required"); return SB_ERR_INVALID_ARG; }
  if ((c->num_pages > 0 && (!c->k || !c->v)) || (c->max_pages > 0 && !c->page_table)) { set_error("pages without an address"); return SB_ERR_INVALID_ARG; }
  return SB_OK;
}
PagedCache make_paged(const sb_cache* c) {
  return PagedCache{c->k, c->v, c->page_table, c->num_pages, c->max_pages, c->page_size, __builtin_ctz((unsigned)c->page_size), c->num_kv_heads};
}

static int check_cache_attn(const sb_cache* c, const sb_chunk* n, int32_t window, int32_t sinks) {
  const int rc = check_cache(c, n);
  if (rc != SB_OK) return rc;
  if (window < 1 || sinks < 0) { set_error("window (%d) must be at least 1 and sinks (%d) not negative", window, sinks); return SB_ERR_INVALID_ARG; }
  return check_rows(n->total_new, n->num_q_heads / c->num_kv_heads);
}

}  // namespace sb

using namespace sb;

extern "C" {

int sb_cache_attn_ws_bytes(const sb_cache* c, const sb_chunk* n, int32_t window, int32_t sinks, int64_t* bytes) {
  if (!bytes) { set_error("null output"); return SB_ERR_INVALID_ARG; }
  const int rc = check_cache_attn(c, n, window, sinks);
  if (rc != SB_OK) return rc;
  *bytes = 0;
  return SB_OK;
}

int sb_cache_attn(const sb_cache* c, const sb_chunk* n, int32_t window, int32_t sinks, const void* q, void* o, float* lse, void* ws, void* stream) {
  int rc = check_cache_attn(c, n, window, sinks);
  if (rc != SB_OK) return rc;
  if (n->total_new == 0 || n->num_seqs == 0 || n->max_new == 0) return SB_OK;
  if (!q || !o || !lse) { set_error("null argument"); return SB_ERR_INVALID_ARG; }
  if ((rc = check_cache_arrays(c, n)) != SB_OK) return rc;
  WindowParams P{};
  P.q = q; P.o = o; P.lse = lse; P.cu = n->cu_new; P.cached = n->cached; P.max_new = n->max_new;
  P.T = n->total_new; P.S = n->num_seqs; P.Hq = n->num_q_heads; P.Hkv = c->num_kv_heads; P.G = P.Hq / P.Hkv;
  P.window = window; P.sinks = sinks;
  P.scale = n->softmax_scale > 0.f ? n->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
  P.scale_log2e = P.scale * 1.4426950408889634f;
  P.cache = make_paged(c);
  KernelTimer kt(K_CACHE_ATTN, (hipStream_t)stream);
  return launch_window_fwd(P, c->head_dim, c->dtype, true, row_tiles_most(P.T, P.S, P.G, forward_rows(c->dtype)), (hipStream_t)stream);
}

}  // extern "C"
