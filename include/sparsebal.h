/*
 * libsparsebal — packed (varlen), causal, GQA dynamic block-sparse attention, forward and
 * backward, with a per-sequence sparsity budget.  MI355X (gfx950) only.
 *
 * The computation is the block-sparse attention of the SparseBalance paper (arXiv 2604.13847),
 * section 2.2: keys/values are cut into fixed-size blocks, a routing score relates each query
 * block to the mean of each key block (the MoBA indexer the paper reuses), the Top-K blocks are
 * kept, and attention is one softmax over the kept keys (Eq. 2; Eq. 1 when every block is kept).
 * The budget k (number of kept blocks) is set per sequence, which is what the paper's dynamic
 * sparsity tuning (section 4.1, Algorithm 1 output) feeds into the kernel.
 *
 * Conventions
 *   - Every function returns SB_OK (0) or a negative error; sb_last_error() gives thread-local text.
 *   - "dev" pointers are device (HBM) addresses, "host" pointers are host addresses.
 *   - The caller owns every buffer, including workspaces; the library never allocates or frees
 *     device memory and never synchronises the stream.  All device work is enqueued on the
 *     hipStream_t passed as `stream` (a null pointer is the default stream).  Host arrays are read
 *     during the call only.
 *   - Layouts are row-major and contiguous, last index fastest:
 *       Q, O, dO, dQ : [T][Hq][D]     K, V, dK, dV : [T][Hkv][D]     LSE : [Hq][T] float
 *     Block j of sequence s covers packed rows cu[s]+j*B .. min(cu[s]+(j+1)*B, cu[s+1])-1; blocks
 *     are aligned to the sequence start and never straddle sequences.
 *     n_s = ceil(L_s/B) blocks per sequence, NQB = sum_s n_s, qb_off[s] = sum_{t<s} n_t.
 *   - Selection heads Hs: Hq in SB_SELECT_PER_QHEAD (one block list per query head) or Hkv in
 *     SB_SELECT_PER_KVGROUP (one list shared by the Hq/Hkv query heads of a KV head; its score is
 *     the sum of their scores).  Query head h reads KV head h / (Hq/Hkv).
 *   - scores: per sequence a dense [Hs][n_s][n_s] float block at element offset Hs*sum_{t<s} n_t^2;
 *     entry (hs,i,j) with j >= i is -infinity.
 *   - Selection CSR: row id = hs*NQB + qb_off[s] + i has c(s,i) = min(k_s, i+1) entries, the block
 *     indices (local to the sequence) kept by query block i, ascending, the last being i itself.
 *     sel_rowptr is therefore a closed form of cu_seqlens and topk.
 *   - No call takes the size of a buffer: every `ws`, `plan` and output must have at least the size sb_get_layout
 *     reports for the same problem; an undersized buffer is overrun, not detected.
 *   - A `ws` buffer is scratch of one call at a time (tables, counters, converted operands): calls that may overlap in
 *     time (different streams) need buffers of their own; calls ordered on one stream may share one.  The library keeps
 *     no device state between calls besides what `plan` and `ws` hold (and the built-in scratch of sb_select_topk_static).
 *   - Supported: block_size 64, 128 or 256; head_dim 64 or 128; Hq % Hkv == 0; n_s <= SB_MAX_BLOCKS_PER_SEQ;
 *     in SB_SELECT_PER_KVGROUP Hq/Hkv <= 8; selection entries and rows (at the granularity of 64-token tiles) must
 *     fit 32-bit row pointers.  Anything else returns SB_ERR_UNSUPPORTED.
 *   - Degenerate inputs: empty sequences are allowed; T == 0 or S == 0 is a no-op returning SB_OK;
 *     k_s > n_s is clamped to n_s; k_s < 1 is an error.
 */
#ifndef SPARSEBAL_H
#define SPARSEBAL_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SB_OK 0
#define SB_ERR_INVALID_ARG (-1)
#define SB_ERR_UNSUPPORTED (-2)
#define SB_ERR_WORKSPACE_TOO_SMALL (-3) /* sb_select_topk_static: the problem's tables exceed the built-in scratch */
#define SB_ERR_HIP (-4)

#define SB_BF16 0 /* Q,K,V,O,dO,dQ,dK,dV are bfloat16 */
#define SB_F32 1  /* they are float; the attention kernels round them to bfloat16 on entry */

#define SB_SELECT_PER_QHEAD 0
#define SB_SELECT_PER_KVGROUP 1

#define SB_MAX_BLOCKS_PER_SEQ 16384

typedef struct sb_problem {
  int32_t total_tokens, num_seqs;          /* T, S */
  int32_t num_q_heads, num_kv_heads;       /* Hq, Hkv */
  int32_t head_dim, block_size;            /* D, B */
  int32_t dtype;                           /* SB_BF16 | SB_F32 */
  int32_t select_mode;                     /* SB_SELECT_PER_QHEAD | SB_SELECT_PER_KVGROUP */
  float softmax_scale;                     /* the 1/sqrt(d) of Eq. 1-2; <= 0 means 1/sqrt(head_dim) */
  float score_scale;                       /* factor on the routing score; <= 0 means softmax_scale */
  const int32_t *cu_seqlens_host;          /* host [S+1], cu[0] = 0, non-decreasing, cu[S] = T */
  const int32_t *cu_seqlens_dev;           /* dev  [S+1], same values */
  const int32_t *topk_host;                /* host [S], budget k_s >= 1 counting the diagonal block */
  const int32_t *topk_dev;                 /* dev  [S], same values */
} sb_problem;

/* Sizes a caller needs before allocating; filled on the host from sb_problem alone. */
typedef struct sb_layout {
  int64_t num_qblocks;   /* NQB */
  int64_t sel_heads;     /* Hs */
  int64_t scores_elems;  /* floats in `scores` */
  int64_t pooled_elems;  /* floats in `kbar_out`: NQB*Hkv*D */
  int64_t sel_rows;      /* Hs*NQB; sel_rowptr holds sel_rows+1 int32 */
  int64_t sel_nnz;       /* int32 entries in sel_idx */
  int64_t plan_bytes;    /* bytes of the `plan` buffer of sb_plan_worklist */
  int64_t scores_ws_bytes, select_ws_bytes, fwd_ws_bytes, bwd_ws_bytes; /* bytes of the `ws` arguments */
  int64_t attended_pairs_per_head_sum; /* sum over query heads of unmasked (query,key) pairs,
                                          the diagonal block counted as its causal triangle */
  int64_t coverage_ws_bytes; /* bytes of the `ws` argument of sb_score_coverage */
} sb_layout;

/* Host only.  Validates the problem and fills `out`. */
int sb_get_layout(const sb_problem *p, sb_layout *out);

/* Host only.  Budget from a keep ratio: k_s = clamp(ceil(rho_s*n_s - 1e-6), 1, n_s), one budget per
 * sequence (the budget is a count of selected blocks, paper section 2.2). */
int sb_keep_ratio_to_topk(const int32_t *cu_seqlens_host, int32_t S, int32_t block_size,
                          const float *keep_ratio_host, int32_t *topk_out_host);

/* Host only.  Writes the closed-form CSR row pointers (sel_rows+1 int32) to a host array. */
int sb_sel_rowptr_host(const sb_problem *p, int32_t *rowptr_out_host);

/* Routing scores (paper section 2.2, MoBA indexer): score[s][hs][i][j] = score_scale *
 * < mean of Q over query block i , mean of K over key block j > for j < i (summed over the group's
 * query heads in SB_SELECT_PER_KVGROUP), -infinity for j >= i.  Means are over the valid tokens of a
 * block.  q, k: dev, dtype per p->dtype.  kbar_out: dev [NQB][Hkv][D] float or null.  scores_out:
 * dev, scores_elems floats.  ws: dev, scores_ws_bytes. */
int sb_block_scores(const sb_problem *p, const void *q, const void *k, float *kbar_out, float *scores_out,
                    void *ws, void *stream);

/* Top-K block selection (paper section 2.2): for every row (s,hs,i) keep the diagonal block i plus
 * the c(s,i)-1 best past blocks j < i under the total order (score descending, then block index
 * ascending; -0 == +0; NaN below every number).  Bit-exact function of `scores`.  Writes
 * sel_rowptr_out (dev, sel_rows+1 int32) and sel_idx_out (dev, sel_nnz int32).  ws: dev, select_ws_bytes. */
int sb_select_topk(const sb_problem *p, const float *scores, int32_t *sel_rowptr_out, int32_t *sel_idx_out,
                   void *ws, void *stream);

/* sb_select_topk for callers that cannot allocate device memory or bring a workspace: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments minus `ws`, same results bit for bit.  The
 * geometry tables that `ws` holds in sb_select_topk (problems of more than 64 sequences need them) live in a device array built
 * into the library (SB_STATIC_SELECT_WS_BYTES per GPU, held until the process ends); a problem whose tables (select_ws_bytes of
 * sb_layout) would not fit returns SB_ERR_WORKSPACE_TOO_SMALL and enqueues nothing, whatever its number of sequences.  The call
 * allocates and frees nothing.  All calls on one GPU share that array: calls on different streams of one GPU that overlap in time
 * race unless both have at most 64 sequences; calls on one stream are ordered.  The first
 * call on a device looks up the array's address (a host-side query, no allocation); make it outside graph capture. */
#define SB_STATIC_SELECT_WS_BYTES (1 << 20)
int sb_select_topk_static(const sb_problem *p, const float *scores, int32_t *sel_rowptr_out, int32_t *sel_idx_out,
                          void *stream);

/* The indexer and the Top-K selection as one step (paper section 2.2).  Arguments as for
 * sb_block_scores and sb_select_topk; ws: dev, scores_ws_bytes.  sel_rowptr_out and sel_idx_out are
 * bit-identical to calling the two separately, whichever form is used:
 *   scores_out != NULL  the score matrix is written as by sb_block_scores (it stays available for the
 *                       budget controller below) and the selection is taken from it (small problems: one kernel
 *                       writes it and selects);
 *   scores_out == NULL  one kernel computes each row's scores on chip and selects there: the score
 *                       matrix (scores_elems floats) is neither allocated nor written nor read back.
 *                       A sequence so long that a single row of keys does not fit the compute unit's
 *                       local memory returns SB_ERR_UNSUPPORTED (not reachable below
 *                       SB_MAX_BLOCKS_PER_SEQ on gfx950). */
int sb_score_select(const sb_problem *p, const void *q, const void *k, float *kbar_out, float *scores_out,
                    int32_t *sel_rowptr_out, int32_t *sel_idx_out, void *ws, void *stream);

/* Work plan for the attention kernels: query-major work items (s,hs,i) ordered by decreasing
 * selected-block count (longest first, as in balanced partitioning by workload weight, paper
 * section 4.3), the key-major transpose of the selection (for every (s,hs,j) the set of query
 * blocks that kept j) and key-major items ordered by decreasing weight; a column that very many query blocks
 * kept (an attention sink) is cut into several items of bounded weight, and in small problems heavy items are walked by
 * several workgroups, so that no single workgroup becomes the straggler the paper's section 3.2 describes.  plan_out: dev, plan_bytes, opaque; it is valid for this problem and
 * this selection only. */
int sb_plan_worklist(const sb_problem *p, const int32_t *sel_rowptr, const int32_t *sel_idx, void *plan_out,
                     void *stream);

/* Host only; for tests and tools that check the plan's properties (every item once, longest first, the transpose is a
 * transpose).  Writes byte offsets into the plan buffer and three sizes to out[SB_PLAN_NUM_SECTIONS]:
 *   QB_OFF   int32 [S+1]      first 64-token tile of every sequence
 *   BM_OFF   int64 [S+1]      first bitmap word of every sequence (per selection head), n_s * ceil(n_s/32) words each
 *   QB_SEQ   int32 [NQB]      sequence of every tile
 *   WORK_FWD int32 [Hs*NQB]   selection rows (hs * NQB + tile) in launch order, longest first
 *   COLCOST  int32 [Hkv*NQB]  (query block, query head) tiles of every key-major column g * NQB + tile
 *   BITMAP   uint32           bit i of word (s, hs, j, i/32): query tile i of head hs kept key tile j
 *   BWD_ITEMS 4 x int32 each  key-major items in launch order: column (or -1: none), bitmap words lo | hi << 16 the item
 *                             covers, partial slot (or -1: the item is the whole column), tiles; BWD_ITEMS_COUNT entries
 *   COUNTERS int32 [3]        partial slots in use, split columns, further slots in use for items that several workgroups walk
 *   SPLIT_COLS 3 x int32 each column, first partial slot, parts
 *   SPLIT_WEIGHT              a column with more tiles than this is cut into parts of at least this many
 * (NQB counts 64-token tiles, whatever the selection block size.) */
#define SB_PLAN_QB_OFF 0
#define SB_PLAN_BM_OFF 1
#define SB_PLAN_QB_SEQ 2
#define SB_PLAN_WORK_FWD 3
#define SB_PLAN_COLCOST 4
#define SB_PLAN_BITMAP 5
#define SB_PLAN_BWD_ITEMS 6
#define SB_PLAN_COUNTERS 7
#define SB_PLAN_SPLIT_COLS 8
#define SB_PLAN_BWD_ITEMS_COUNT 9
#define SB_PLAN_SPLIT_WEIGHT 10
#define SB_PLAN_SPLIT_MAX 11
#define SB_PLAN_NUM_SECTIONS 12
int sb_plan_sections(const sb_problem *p, int64_t *out);

/* Forward (Eq. 2): for every query row r of query block i and query head h,
 * O_r = sum_j softmax_j(softmax_scale * q_r.k_j) v_j over the keys j of the selected blocks that are
 * not in r's future; LSE_r = log sum_j exp(softmax_scale * q_r.k_j).  Any valid selection is
 * accepted (ascending, unique, <= i, containing i).  o: dev like q; lse: dev [Hq][T] float;
 * ws: dev, fwd_ws_bytes. */
int sb_sparse_attn_fwd(const sb_problem *p, const void *q, const void *k, const void *v,
                       const int32_t *sel_rowptr, const int32_t *sel_idx, const void *plan, void *o, float *lse,
                       void *ws, void *stream);

/* Backward of Eq. 2 with the selection held fixed: dQ, dK, dV from dO (dK, dV summed over the
 * query heads of each KV head).  o and lse are the forward's outputs.  Deterministic: every output
 * element is accumulated in a fixed order, by one workgroup or as partial sums of several that are
 * added in a fixed order.  ws: dev, bwd_ws_bytes. */
int sb_sparse_attn_bwd(const sb_problem *p, const void *q, const void *k, const void *v, const void *o,
                       const float *lse, const void *d_o, const int32_t *sel_rowptr, const int32_t *sel_idx,
                       const void *plan, void *dq, void *dk, void *dv, void *ws, void *stream);

/* ---- budget controller (paper sections 4.1 and 4.2): what sets topk[] before the calls above ----
 *
 * Coverage curves of the routing scores (section 4.1, Eq. 4).  For query block i of sequence s and one
 * selection head, the scores of the earlier blocks j < i are normalised by a softmax and sorted in
 * descending order into importance scores r_1 >= r_2 >= ... (sum 1); a budget k keeps the diagonal
 * block plus the k-1 best earlier blocks, so the row covers the sum of its min(k-1, i) largest r.
 * C_s(k), k = 1..n_s, is the mean of that over the sequence's query blocks and selection heads:
 * non-decreasing, C_s(1) = 1/n_s, C_s(n_s) = 1.  `scores`: dev, as written by sb_block_scores (finite
 * for j < i).  coverage_out: dev, NQB floats, C_s(k) at qb_off[s] + k - 1.  ws: dev, coverage_ws_bytes.
 * Deterministic (fixed summation order). */
int sb_score_coverage(const sb_problem *p, const float *scores, float *coverage_out, void *ws, void *stream);

/* Profiled latency table M[x, k] (section 4.2, Eq. 10): latency[a*num_budgets + b] is the measured
 * latency at length lengths[a] (tokens) and budget budgets[b] (blocks); both grids strictly
 * increasing.  All pointers are host pointers; the caller owns them. */
typedef struct sb_perf_table {
  int32_t num_lengths, num_budgets;
  const float *lengths;
  const float *budgets;
  const float *latency;
} sb_perf_table;

/* Host only.  Perf.predict (Eq. 8): the table interpolated linearly in length and in budget, clamped
 * at its edges. */
int sb_perf_predict(const sb_perf_table *t, double length, double budget, double *latency_out);

/* Host only.  Perf.align (Eq. 9): the largest integer budget in 1..max_budget whose predicted latency
 * does not exceed target_latency; 1 if none does. */
int sb_perf_align(const sb_perf_table *t, double length, double target_latency, int32_t max_budget,
                  int32_t *budget_out);

/* Host only.  Workload-aware dynamic sparsity tuning (section 4.1, Algorithm 1) with every packed
 * sequence as one micro-batch.  p->topk_host are the base budgets k_base.  T_anchor is the minimum,
 * mean or maximum (Eq. 3) of the predicted latencies at the base budgets; k_anchor = Perf.align(L_s,
 * T_anchor) in 1..n_s; the final budget is k_anchor unless C_s(k_base) - C_s(k_anchor) exceeds
 * threshold_p (Eq. 5), in which case it is the smallest k with C_s(k_base) - C_s(k) <= threshold_p.
 * coverage_host: host copy of sb_score_coverage's output.  topk_final_out: host [S];
 * topk_anchor_out (host [S]) and t_anchor_out may be null.  Empty sequences keep their base budget. */
#define SB_ANCHOR_MIN 0
#define SB_ANCHOR_MEAN 1
#define SB_ANCHOR_MAX 2
int sb_dst_tune(const sb_problem *p, const float *coverage_host, const sb_perf_table *perf, int anchor,
                double threshold_p, int32_t *topk_final_out, int32_t *topk_anchor_out, double *t_anchor_out);

/* ---- sparsity-aware batching (paper section 4.3, Algorithm 2); host only, CPU side of the data loader ----
 *
 * Sparsity predictor Spar: for each sequence-length bin b (bin_edges[b] <= L < bin_edges[b+1], lengths
 * outside clamp to the first / last bin) an exponential moving average of the final budgets the
 * tuning step produced: ema[b] <- decay*ema[b] + (1-decay)*k per sample, in order; the first sample of
 * a bin initialises it (seen[b] = 1).  sb_spar_predict returns ema[b], or k_base while the bin has
 * seen nothing.  ema: [num_bins] float, seen: [num_bins] bytes, bin_edges: [num_bins+1]; caller-owned. */
int sb_spar_update(float *ema, uint8_t *seen, const float *bin_edges, int32_t num_bins, double decay,
                   const int32_t *lengths, const int32_t *k_final, int32_t n);
int sb_spar_predict(const float *ema, const uint8_t *seen, const float *bin_edges, int32_t num_bins,
                    int32_t length, double k_base, double *k_out);

/* `bin_packing`: balanced partition of n weights into num_bins bins by the longest-first greedy
 * (decreasing weight, ties to the lower index; each to the least loaded bin, ties to the lower bin).
 * bin_of_out[i] is the bin of sample i.  Bin sizes are not constrained. */
int sb_balanced_partition(const double *weights, int32_t n, int32_t num_bins, int32_t *bin_of_out);

/* Algorithm 2: W[i] = Perf.predict(lengths[i], k_pred[i]); samples are split over dp_size DP ranks, then
 * the samples of dp_rank over num_microbatches micro-batches (= gbs / (mbs * N)).  weights_out (nullable),
 * dp_bin_out, mb_bin_out: [n]; mb_bin_out is -1 for the samples of other ranks. */
int sb_sab_batches(const sb_perf_table *perf, const int32_t *lengths, const double *k_pred, int32_t n,
                   int32_t dp_size, int32_t dp_rank, int32_t num_microbatches, double *weights_out,
                   int32_t *dp_bin_out, int32_t *mb_bin_out);

/* ---- rotary positions ----
 *
 * Turns the first rot_dim elements of every head of q and k by the token's position: pair i of a head, (x, y) = elements (i, i + rot_dim/2)
 * in SB_ROPE_HALF or (2i, 2i + 1) in SB_ROPE_INTERLEAVED, becomes amplitude * (x cos a - y sin a, y cos a + x sin a) with
 * a = 2 pi * position * turns[i]; elements from rot_dim on are copied.  Angles are reduced in 64 bits, so that far positions lose nothing.
 *
 * sb_rope is plain data that the caller keeps; sb_rope_init fills it, a caller with frequencies of its own may write `turns` (revolutions per
 * token, pairs 0 .. rot_dim/2 - 1) and `amplitude` itself. */
#define SB_ROPE_HALF 0
#define SB_ROPE_INTERLEAVED 1
#define SB_ROPE_PLAIN 0  /* f_i = base^(-2i/rot_dim) radians per token */
#define SB_ROPE_LINEAR 1 /* f_i / factor */
#define SB_ROPE_NTK 2    /* base * factor^(rot_dim/(rot_dim-2)) in place of base */
#define SB_ROPE_YARN 3   /* f_i / factor for pairs that turn less than `low` times in original_length tokens, f_i for those that turn more than
                            `high` times, between the two linear in i (bounds rounded outwards to whole pairs); amplitude 0.1 ln(factor) + 1 */
#define SB_ROPE_BANDS 4  /* likewise, linear in the number of turns, amplitude 1 */
#define SB_ROPE_MAX_PAIRS 64
typedef struct sb_rope {
  int32_t rot_dim; /* even, 2 .. head_dim */
  int32_t layout;  /* SB_ROPE_HALF | SB_ROPE_INTERLEAVED */
  float amplitude;
  int32_t reserved;
  double turns[SB_ROPE_MAX_PAIRS];
} sb_rope;

/* Host only.  rot_dim even, 2 .. 2*SB_ROPE_MAX_PAIRS (SB_ROPE_NTK: from 4 on); base > 1; factor >= 1 (read from SB_ROPE_LINEAR on);
 * original_length > 0, low, high (read by SB_ROPE_YARN and SB_ROPE_BANDS; low, high <= 0 mean 1 and 32, or 1 and 4; low < high). */
int sb_rope_init(sb_rope *out, int32_t rot_dim, int32_t layout, double base, int32_t scaling, double factor, double original_length,
                 double low, double high);

/* q_out, k_out (contiguous) from q, k, whose tokens lie q_pitch and k_pitch elements apart (0: contiguous, else at least H*D; a slice of a
 * fused projection); dtype per p->dtype.  positions: dev int32 [T], or null for the token's index in its sequence.  direction SB_ROPE_FORWARD
 * turns by the angle, SB_ROPE_BACKWARD by its negative, which makes gradients of q and k from those of q_out and k_out.  q or k may be
 * null together with its output.  An output may be its own input (contiguous); other overlaps are not allowed.  Of `p` this reads
 * total_tokens, num_seqs, the heads, head_dim, dtype and cu_seqlens (cu_seqlens_dev only where positions is null); no workspace. */
#define SB_ROPE_FORWARD 0
#define SB_ROPE_BACKWARD 1
int sb_rope_apply(const sb_problem *p, const sb_rope *r, const int32_t *positions, const void *q, int64_t q_pitch, const void *k,
                  int64_t k_pitch, void *q_out, void *k_out, int direction, void *stream);

/* Positions with several axes (time, height and width of image and video tokens): pair i turns by the position on axis axis[i], so
 * a = 2 pi * positions[axis[i]][token] * turns[i].
 *
 * sb_rope_axes is plain data like sb_rope; sb_rope_axes_init fills it from how many pairs each axis has: SB_AXES_SECTIONS, the first pairs are axis 0's, the next
 * ones axis 1's; SB_AXES_IN_TURN, pairs are dealt to axes 0, 1, .., num_axes - 1, 0, 1, .. and an axis that has all of its pairs is left out.  Frequencies stay those of the
 * rope.  Where each axis has frequencies of its own that start anew, sb_rope_join puts the axes' ropes one behind the other (SB_AXES_SECTIONS then): rot_dim is the sum, layout and
 * amplitude have to be the same in all. */
#define SB_ROPE_MAX_AXES 8
#define SB_AXES_SECTIONS 0
#define SB_AXES_IN_TURN 1
typedef struct sb_rope_axes {
  int32_t num_axes;                  /* 1 .. SB_ROPE_MAX_AXES */
  uint8_t axis[SB_ROPE_MAX_PAIRS];   /* of pairs 0 .. rot_dim/2 - 1, below num_axes */
} sb_rope_axes;

/* Host only.  pairs: host [num_axes], none negative, at least one and at most SB_ROPE_MAX_PAIRS in all. */
int sb_rope_axes_init(sb_rope_axes *out, int32_t num_axes, const int32_t *pairs, int32_t order);
/* Host only.  `out` may be one of the ropes. */
int sb_rope_join(sb_rope *out, const sb_rope *ropes, int32_t num_ropes);

/* sb_rope_apply with positions of several axes: dev int32 [num_axes][T].  cu_seqlens is not read on the device. */
int sb_rope_axes_apply(const sb_problem *p, const sb_rope *r, const sb_rope_axes *axes, const int32_t *positions, const void *q, int64_t q_pitch,
                       const void *k, int64_t k_pitch, void *q_out, void *k_out, int direction, void *stream);

/* ---- attention with a sliding window and sinks ----
 *
 * Causal attention of the same packed batches at the granularity of tokens: row t of a sequence sees the keys u <= t with t - u < window or
 * u < sinks (the window counts the row itself, the sinks are the first tokens of the row's sequence).  window >= 1, sinks >= 0; a window of at
 * least the longest sequence is dense causal attention.  O, LSE and the gradients are those of sb_sparse_attn_fwd / _bwd with these keys
 * in place of the selected ones.  Of `p` this reads total_tokens, num_seqs, the heads, head_dim, dtype, softmax_scale and cu_seqlens (both
 * copies); block_size, select_mode and the budgets are not read and may be anything.  SB_F32 tensors are computed in float32 throughout (matrix
 * instructions of that type), not rounded to bfloat16.  Non-finite values: NaN and +infinity among the scores that a row sees make its O and
 * LSE NaN.  What the mask hides has weight zero in products that take whole tiles (counted from the sequence's start), and zero times no number is none.
 * So a V that is not finite (in the backward a K too) may reach O and dQ of rows that see any key of its 64-token tile, and of rows up to 31 tokens from such;
 * and a row whose Q, O, LSE or dO is not finite may reach dK and dV of all keys of a 128-token block that it sees any key of: with sinks, of all keys of
 * the block that they are in, from every later row.  It reaches nothing else, and no other sequence or KV head.  A row whose scores are all -infinity has O and LSE NaN.
 * Deterministic.  Tensors and ws start at multiples of 16 bytes; T * Hq/Hkv fits 31 bits.  ws: dev, sizes from sb_window_ws_bytes (host only; either output
 * may be null); of zero bytes it may be null. */
int sb_window_ws_bytes(const sb_problem *p, int32_t window, int32_t sinks, int64_t *fwd_bytes_out, int64_t *bwd_bytes_out);
int sb_window_attn_fwd(const sb_problem *p, int32_t window, int32_t sinks, const void *q, const void *k, const void *v, void *o, float *lse,
                       void *ws, void *stream);
int sb_window_attn_bwd(const sb_problem *p, int32_t window, int32_t sinks, const void *q, const void *k, const void *v, const void *o,
                       const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *ws, void *stream);

/* ---- a paged cache of keys and values, and attention of new tokens over it (serving) ----
 *
 * Tokens j*page_size .. (j+1)*page_size - 1 of sequence s live in page page_table[s][j].  An entry outside 0 .. num_pages - 1 is no page: nothing
 * is written there and its keys are seen by no row; so are tokens from max_pages*page_size on.  Nothing of a page behind the sequence's last token is
 * used, whatever it holds.  Pages may be shared between sequences; one that sb_cache_append writes to belongs to one sequence, and stands in its row
 * once.  All sizes that change from step to step are on the device, so that a captured graph can be replayed with other lengths within max_new and
 * max_pages.  Tensors, pages and ws start at multiples of 16 bytes. */
typedef struct sb_cache {
  int32_t num_pages, page_size; /* page_size: a power of two, 16 .. 1024 */
  int32_t num_kv_heads, head_dim, dtype; /* head_dim 64 or 128; SB_BF16 | SB_F32 */
  int32_t max_pages;            /* entries of a row of page_table */
  void *k, *v;                  /* dev [num_pages][num_kv_heads][page_size][head_dim] */
  const int32_t *page_table;    /* dev [num_seqs][max_pages] */
} sb_cache;
typedef struct sb_chunk {       /* the new tokens of num_seqs sequences, packed: rows cu_new[s] .. cu_new[s+1] - 1 are those of sequence s */
  int32_t num_seqs, num_q_heads;
  int32_t total_new;            /* rows of q, k, v and the outputs.  Rows from cu_new[num_seqs] on belong to no sequence and are left as they were */
  int32_t max_new;              /* no sequence has more new tokens; rows beyond are left as they were */
  int32_t max_length;           /* about how long the longest sequence gets: what the work is split by, no bound */
  float softmax_scale;          /* <= 0 means 1/sqrt(head_dim) */
  const int32_t *cu_new;        /* dev [num_seqs+1], non-decreasing */
  const int32_t *cached;        /* dev [num_seqs]: tokens in front of the new ones */
} sb_chunk;

/* Writes the new tokens' k (turned by their positions cached[s] + i, unless r is null) and v into their pages, and q turned likewise to q_out.
 * k, v: dev [total_new][Hkv][D], tokens k_pitch, v_pitch elements apart (0: contiguous); q: [total_new][Hq][D] with q_pitch, or null together with q_out (contiguous). */
int sb_cache_append(const sb_cache *c, const sb_chunk *n, const sb_rope *r, const void *q, int64_t q_pitch, const void *k, int64_t k_pitch,
                    const void *v, int64_t v_pitch, void *q_out, void *stream);

/* sb_cache_append with positions of several axes: dev int32 [num_axes][total_new].  What a token turns by is theirs; where it is kept, and what it sees, still goes by cached[s] + i. */
int sb_cache_append_axes(const sb_cache *c, const sb_chunk *n, const sb_rope *r, const sb_rope_axes *axes, const int32_t *positions, const void *q, int64_t q_pitch,
                         const void *k, int64_t k_pitch, const void *v, int64_t v_pitch, void *q_out, void *stream);

/* Attention of the new tokens over the cache, which holds them already (sb_cache_append): row i of sequence s is token t = cached[s] + i and sees
 * the keys u <= t with t - u < window or u < sinks.  Non-finite values as in sb_window_attn_fwd.  q, o: dev [total_new][Hq][D]; lse: dev [Hq][total_new] float.  A row that sees no key (its
 * pages are missing), or only keys whose scores are -infinity, has O = 0 and LSE = -infinity.  From one token to whole prompts.  ws: dev, sb_cache_attn_ws_bytes (host only). */
int sb_cache_attn_ws_bytes(const sb_cache *c, const sb_chunk *n, int32_t window, int32_t sinks, int64_t *bytes_out);
int sb_cache_attn(const sb_cache *c, const sb_chunk *n, int32_t window, int32_t sinks, const void *q, void *o, float *lse, void *ws, void *stream);

/* ---- page tables built on the GPU ----
 *
 * A pool of pages and the tables of the sequences that hold them, all on the device.  Row s of page_table holds the sequence's pages in entries 0 .. held[s] - 1 and
 * -1 behind them; a page that no row holds is one of free_pages[0 .. free_count - 1], a stack.  The caller fills them once (free_pages with all pages, free_count
 * num_pages, held 0, the table -1), and sb_cache_tables keeps them: after the call row s holds as many pages as its tokens take, ceil(length / page_size), at most max_pages,
 * where its length is cached[s] + added[s], or 0 where added[s] < 0 (the sequence is finished).  Entries that are too many go back first, the last entry of the last
 * row before all others; then the rows' missing entries are filled in order from the stack's top.  So two calls that undo each other's lengths (room for drafted tokens,
 * and the end of those that were rejected) leave everything as it was.  Where pages run out, the first rows get them; missing_out (dev, may be null) is how many lacked.
 * Negative `cached` counts as 0; held and free_count outside what the arrays hold are taken as the nearest value inside.  Rows own their pages: none stands in two rows.
 *
 * Also written, all of the call's new tokens packed as in sb_chunk: cu_new_out dev [num_seqs+1] (of max(added, 0); sums stop at 2^31 - 1); and, each unless null, for tokens
 * 0 .. total_new - 1 positions_out dev int32 (cached[s] + i) and slots_out dev int64 (page * page_size + token of the page, -1: no page).  Of tokens behind the last sequence
 * the slot is -1 and the position 0.  total_new is the arrays' size, and with them null it is not read.  cached and added: dev [num_seqs].  No workspace; a captured call serves all steps. */
typedef struct sb_page_pool {
  int32_t num_seqs, max_pages, num_pages;
  int32_t page_size;          /* a power of two, 16 .. 1024 */
  int32_t *page_table;        /* dev [num_seqs][max_pages] */
  int32_t *held;              /* dev [num_seqs] */
  int32_t *free_pages;        /* dev [num_pages] */
  int32_t *free_count;        /* dev [1] */
} sb_page_pool;
int sb_cache_tables(const sb_page_pool *pool, const int32_t *cached, const int32_t *added, int32_t total_new, int32_t *cu_new_out, int32_t *positions_out,
                    int64_t *slots_out, int32_t *missing_out, void *stream);

/* ---- a paged cache in four bits ----
 *
 * The cache of sb_cache_append and sb_cache_attn with keys and values in four bits: 32 neighbouring elements of a head share a step, and an element is that step times 0, 1/2, 1, 3/2,
 * 2, 3, 4 or 6 (codes 0 .. 7; 8 more: negative).  The step is 1/6 of the 32 elements' largest magnitude (their product with the float nearest 1/6), rounded to six significant bits (and a multiple of 2^-131; halves
 * away from zero) and at most 1.3125 * 2^125; a code is that of the nearest value, ties to the even code, of the largest where an element is beyond it, and 0 where the step is 0 or no number.  So every value held is a bfloat16 number; where it
 * is used nothing is rounded again.  32 elements of which one is no number or infinite are all NaN.  Keys are turned in float64 and rounded to float32 before that, so that codes do
 * not depend on how the turn is computed.
 *
 * Per token and KV head D/2 bytes of codes (the lower half of a byte first) and D/32 steps (bfloat16).  Byte D/8 b + 4 c + e of a key holds elements 32 c + 8 b + 2 e and
 * the next (c < D/32, b < 4, e < 4); byte D/32 i + e of a value holds elements 32 e + i and 32 e + 16 + i (i < 16).  72 bytes at head_dim 128 where bfloat16 takes 256. */
typedef struct sb_cache4 {
  int32_t num_pages, page_size;          /* as in sb_cache */
  int32_t num_kv_heads, head_dim, dtype; /* dtype: of the new tokens, the queries and the output (SB_BF16 | SB_F32); the pages are the same */
  int32_t max_pages;
  void *k, *v;                  /* dev [num_pages][num_kv_heads][page_size][head_dim/2] bytes */
  void *k_step, *v_step;        /* dev [num_pages][num_kv_heads][page_size][head_dim/32] bfloat16 */
  const int32_t *page_table;    /* dev [num_seqs][max_pages] */
} sb_cache4;

/* sb_cache_append (axes and positions null) or sb_cache_append_axes into such pages.  r may be null only without axes.  k_held, v_held (dev, contiguous, [total_new][Hkv][D] in c->dtype, or null): the
 * values as they are held from now on, for attention over the packed tokens of a first prompt.  q_out, k_held and v_held lie apart from each other, from all inputs and from the pages (checked); so do
 * the pages from q, k, v and the other inputs, and the cache's arrays from each other (not checked). */
int sb_cache4_append(const sb_cache4 *c, const sb_chunk *n, const sb_rope *r, const sb_rope_axes *axes, const int32_t *positions, const void *q, int64_t q_pitch, const void *k,
                     int64_t k_pitch, const void *v, int64_t v_pitch, void *q_out, void *k_held, void *v_held, void *stream);

/* sb_cache_attn over such pages: the same rows, mask and outputs.  In SB_BF16 probabilities are rounded to bfloat16 once for the product with V; in SB_F32 queries and probabilities are taken as
 * three bfloat16 numbers that add up to them, so that products are exact but for 2^-24 (of values above 2^-100).  A step that is no number makes the rows that see it NaN: of a key their O and LSE, of
 * a value (with a probability above 0) the 32 elements of O that share it.  What the mask hides from a row reaches it nowhere, whatever it holds, in SB_F32 and where min(max_new, total_new) * Hq/Hkv is at most
 * 64; in longer chunks a value's step that is no number may reach O of rows that see any key of its tile of 64 keys (counted from the sequence's start), and of rows up to 31 tokens from such, in its KV
 * head.  ws: dev, sb_cache4_attn_ws_bytes (host only). */
int sb_cache4_attn_ws_bytes(const sb_cache4 *c, const sb_chunk *n, int32_t window, int32_t sinks, int64_t *bytes_out);
int sb_cache4_attn(const sb_cache4 *c, const sb_chunk *n, int32_t window, int32_t sinks, const void *q, void *o, float *lse, void *ws, void *stream);

/* Instrumentation (measurement only; off by default).  `flag` is a bit set:
 *   SB_INSTR_CU_BUSY  the attention kernels add, for every workgroup, its run time in ticks of the
 *                     100 MHz constant clock to a per-compute-unit slot inside `ws`; sb_read_cu_busy
 *                     copies the SB_CU_SLOTS slots of the last forward or backward call that used
 *                     `ws` to host memory (it synchronises the stream).  This is the per-CU busy time
 *                     whose max/mean is the imbalance measure of the paper's Eq. 11 applied to CUs.
 *   SB_INSTR_KERNEL_EVENTS  every kernel launch is bracketed by HIP events on the launch stream;
 *                     sb_read_kernel_times waits for them, writes per-kernel total milliseconds and
 *                     launch counts (SB_NUM_KERNELS entries each, host) and resets the record.  The
 *                     events are recycled: once a few steps have run, a timed launch creates none.
 * The flag and the event record are process-wide (one mutex guards them): calls from several threads
 * are safe, their records interleave.  bwd_dkv also covers the reduction of split key-major columns. */
#define SB_CU_SLOTS 512
#define SB_INSTR_CU_BUSY 1
#define SB_INSTR_KERNEL_EVENTS 2
#define SB_NUM_KERNELS 15 /* pool, score, topk, plan (and page tables), fwd, bwd_prep, bwd_dq, bwd_dkv, coverage, score_select, rope (and append), window_fwd,
                             window_dq (and what prepares it), window_dkv, cache_attn (in four bits too); bwd_prep is the
                             conversion of float32 inputs in the backward call (nothing for bf16 inputs); score_select is the
                             single kernel of sb_score_select, without scores_out or in small problems */
int sb_set_instrumentation(int flag);
int sb_read_cu_busy(const void *ws, uint64_t *busy_out_host, void *stream);
int sb_read_kernel_times(double *total_ms_host, int64_t *launches_host);

const char *sb_last_error(void);
const char *sb_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SPARSEBAL_H */
