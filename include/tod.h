/*
 * tod.h - C ABI of libtod, an MI355X (gfx950) implementation of the exact
 * kNN / LOF outlier-detection hot path of TOD (Zhao, Chen, Jia; arXiv
 * 2110.14007).
 *
 * The library computes, for query rows X_q and reference rows X_r:
 *   - the k nearest references of every query (the paper's kNN functional
 *     operator = cdist fused with topk, Sections 4.2 and 6.1), exact under
 *     the lexicographic key (distance, reference index), so ties go to the
 *     lower index;
 *   - the kNN-OD outlier score (distance to the k-th neighbour, Table 1);
 *   - the LOF outlier score (Table 1; Breunig et al. 2000, with exactly k
 *     neighbours and lrd = 1 / (mean reach-distance + 1e-10)), or, through
 *     tod_lof_ties, on Breunig's tie-inclusive k-distance neighbourhoods.
 *
 * It follows the paper's provable quantization (Section 5.2): inputs are
 * quantised (fp32 / fp16 / bf16 after centring and power-of-two scaling),
 * distances are evaluated in that precision to shortlist K' candidates per
 * query, a certificate checks that no excluded reference can reach the
 * exact k-th distance, and rows that fail it are recomputed exactly
 * (Section 5.2, step iii).  Distances are fused with selection so the n x n
 * matrix never exists (Section 6.1, operator fusion); queries stream through
 * in blocks and references in splits (Section 6, automatic batching).
 *
 * Conventions shared by every entry point:
 *   - Every data pointer is a DEVICE pointer (HIP), owned by the caller.
 *     Inputs are fp32, row-major, contiguous, 16-byte aligned.
 *   - The library allocates no device memory: the caller passes a workspace
 *     (256-byte aligned).  tod_workspace_size() bytes run the queries in as
 *     few blocks as the planner likes; a smaller workspace makes the kNN
 *     entry points plan smaller query blocks (tod_plan_workspace).
 *   - Distances are Euclidean (not squared).  Index outputs are 0-based rows
 *     of the reference set.  Output rows are sorted by (distance, index).
 *   - Arguments are validated on the host before any HIP call; on an
 *     argument error nothing is launched and outputs are untouched.
 *   - Calls are blocking: they return after the work queued on `stream`
 *     (a hipStream_t, or NULL for the default stream) has finished, so the
 *     returned status is final.  The library keeps no state between calls;
 *     calls on different streams with different workspaces may overlap.
 *   - On any error other than TOD_OK, output contents are unspecified.
 */
#ifndef TOD_H
#define TOD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TOD_OK = 0,
  TOD_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, k out of range, bad struct_size */
  TOD_ERR_NONFINITE = 2,   /* NaN or Inf in the input (the rounding analysis needs finite data) */
  TOD_ERR_WORKSPACE = 3,   /* workspace misaligned, or too small for one 32-row query block */
  TOD_ERR_UNSUPPORTED = 4, /* k > 256, d > 4096, or more than 2^31 - 1 rows */
  TOD_ERR_HIP = 5,         /* a HIP launch or runtime call failed; see tod_last_error() */
  TOD_ERR_INTERNAL = 6,
  TOD_ERR_CAPACITY = 7     /* tod_nwr, tod_loci, tod_lof_ties: more pairs in range than the
                            * output capacity (tod_nwr still writes the row offsets and the
                            * total) */
} tod_status;

/* Precision of the shortlist filter (the exact recheck always works from the
 * original fp32 rows with fp64 accumulation). */
typedef enum {
  TOD_PREC_AUTO = 0,
  TOD_PREC_FP32 = 1, /* fp32 FMA distance tile: the reference filter (shortest shortlist,
                      * fewest fallbacks), not the fast path.  Its vector FMA work has a
                      * floor of 2d flop per pair at the non-packed fp32 rate, 8.1 ms at
                      * n = 100,000, d = 32 against the fp16 tile's 2.2 ms, and it runs at
                      * about 10x the fp16 tile's time. */
  TOD_PREC_FP16 = 2, /* fp16 MFMA distance tile, fp32 accumulate */
  TOD_PREC_BF16 = 3  /* bf16 MFMA distance tile, fp32 accumulate */
} tod_precision;

/* Outlier score from the k exact neighbour distances of a point (the kNN
 * detector of Table 1: the distance to the k-th neighbour, or an aggregate of
 * the k distances such as Angiulli and Pizzuti's weight, their sum). */
typedef enum {
  TOD_SCORE_KTH = 0,    /* distance to the k-th nearest neighbour (default) */
  TOD_SCORE_MEAN = 1,   /* mean of the k distances */
  TOD_SCORE_MEDIAN = 2, /* median of the k distances (mean of the two middle ones for even k) */
  TOD_SCORE_SUM = 3     /* sum of the k distances */
} tod_score;

typedef struct {
  uint32_t struct_size;  /* must be sizeof(tod_options) */
  int32_t precision;     /* tod_precision; AUTO picks by d */
  int32_t exclude_self;  /* tod_knn only: drop reference j == query i (requires xq == xr, nq == nr) */
  int32_t shortlist;     /* K' (candidates per query kept by the filter); 0 = planner */
  int64_t query_block;   /* query rows per block (rounded up to 32); 0 = planner */
  int32_t ref_splits;    /* reference splits processed in parallel; 0 = planner */
  float margin_scale;    /* >= 1: multiplies every error term of the certificate; 1 = default */
  int32_t force_fallback;/* debug: treat every row as uncertified (exact recomputation) */
  int32_t no_recheck;    /* debug: return the filter's shortlist order without verification */
  int32_t reorder;       /* scan order and pruned scan of an X-against-X call (tod_knn with
                          * xq == xr, tod_knn_score, tod_lof, tod_lof_ties, tod_abod, tod_cof)
                          * through the register-list kernel (fp16 / bf16 filter, d <= 512, K' up
                          * to 64, or 128 beyond 128 columns): 0 = planner, 1 = on, -1 = off.
                          * Order: the rows are grouped by their nearest of G evenly spaced rows
                          * (G = 16, or for rows of at most 16 elements one per 8192 rows, up to
                          * 1024) and every query block first scans the references of its own
                          * group, so the filter's thresholds tighten early.
                          * Pruned scan: the order follows the nearest of 16 pivots and the
                          * distance from it (d > 16), or a k-d tree over the columns, and
                          * references whose box lies beyond a wave's K'-th distances are left
                          * out.  Where the boxes rule too little out, the plain scan runs.
                          * Planner: the order from 4096 rows on where the scan has one split;
                          * the pruned scan, in query blocks of 8192 rows and more and with
                          * ref_splits 0 or 1, from 60,000 rows on (d > 16), 65,536 (d <= 6),
                          * 131,072 (d = 7, 8) or 2^20 (d = 9..16; one split).  On: from the first
                          * row.  Results are identical either way. */
  int32_t score;         /* tod_score: the kNN outlier score of tod_knn_score, tod_knn_decision
                          * and tod_lof's knn_score_out */
  int32_t tail_parts;    /* fp16 / bf16 filter with one reference split: the workgroups of a
                          * query block's last, partly filled round of the GPU scan the
                          * references in this many parts on separate workgroups (their lists
                          * are merged before the recheck); 0 = planner, 1 = off, at most 8.
                          * The pruned scan cuts its long scans by a plan of its own into the
                          * same room; with 1 it cuts none, and runs only in blocks of 2^17 rows
                          * and more.  Results are identical either way. */
} tod_options;

/* Plan and per-phase timings of one call (filled when a non-NULL pointer is
 * passed; timings are measured with HIP events on the call's stream). */
/* (The recheck's candidate count m is not reported per call: it grows per
 * row, k + 8 first and then 16 more at a time up to K', so rows_certified and
 * rows_fallback carry what a single maximum would summarise.) */
typedef struct {
  uint32_t struct_size;   /* sizeof(tod_stats), or TOD_STATS_SIZE_1 (without the last three
                           * fields, which such a call leaves alone) */
  int32_t precision;      /* resolved tod_precision */
  int32_t kprime;         /* shortlist length K' */
  int32_t ref_splits;     /* S (with pruned_kind > 0: of the blocks that the plain scan takes) */
  int64_t query_block;    /* B_q */
  int64_t blocks;         /* number of query blocks */
  int64_t rows_certified; /* rows whose shortlist passed the certificate */
  int64_t rows_fallback;  /* rows recomputed exactly */
  int64_t tile_launches;  /* launches of the fused distance + selection kernel that scanned
                           * references (a block with a tail split takes two) */
  float ms_prep, ms_tile, ms_recheck, ms_fallback, ms_score, ms_total;
                          /* ms_recheck includes the merge of the split lists, which runs
                           * inside the recheck kernel (there is no separate ms_merge) */
  int32_t reordered;      /* 1 if the rows were put in the grouped order (see tod_options.reorder) */
  int64_t pairs_candidate; /* range queries (tod_nwr, tod_loci, tod_lof_ties): pairs the filter
                            * could not rule out of range */
  int64_t pairs_uncertain; /* range queries: candidates whose test needed the exact distance */
  int64_t pairs_in_range;  /* range queries: pairs within the threshold */
  int32_t tail_parts;      /* parts the last partly filled round of a plain scan was scanned in
                            * (1: none) */
  int64_t tail_rows;       /* query rows scanned in parts, summed over the blocks */
  int32_t list_runs;       /* 2 if each shortlist was built as two runs of K'/2 entries (the
                            * register-list tile over two pieces of the scan order: K' = 128
                            * on rows of 129..512 elements), else 1 */
  int32_t pruned_kind;     /* boxes of the pruned scan (see tod_options.reorder): 0 none, 1
                            * distances to pivots, 2 columns */
  int64_t pruned_blocks;   /* query blocks that the pruned scan ran; the others' boxes ruled out
                            * too little, and the plain scan took over */
  int64_t pairs_scanned;   /* kNN calls: (query, reference) pairs whose key the filter computed,
                            * counted by 32 queries and 128 references in the pruned scan */
} tod_stats;
/* (pruned_kind lies in the padding that ended the first layout.) */
#define TOD_STATS_SIZE_1 ((uint32_t)offsetof(tod_stats, pruned_blocks))

/* Fill *opts with defaults: AUTO precision (the fp16 filter of Section 5.2's
 * provable quantization), planner-chosen K', query block and splits
 * (Section 6), self pair kept, margin_scale 1. */
void tod_default_options(tod_options* opts);

/*
 * Workspace bytes with which the call runs its queries in as few blocks as
 * the planner likes (Section 6: the batches are sized to the GPU memory at
 * hand; a smaller workspace gives smaller query blocks, see
 * tod_plan_workspace).  One function serves every entry point through
 *   mode 0: tod_knn, tod_knn_score, tod_knn_decision (any query and reference sets);
 *   mode 1: tod_lof, tod_abod, tod_cof (X against itself, nq == nr: these
 *           keep the neighbour lists and the LOF buffers as well);
 *   mode 2: tod_knn_classify (neighbour lists for the vote).
 * (mode is an addition to the interface the kNN/LOF calls alone would need:
 * the detectors built on the same lists need more room.)
 * Returns 0 if the arguments are invalid or unsupported.
 */
size_t tod_workspace_size(int64_t nq, int64_t nr, int64_t d, int32_t k, int32_t mode,
                          const tod_options* opts);

/*
 * kNN: for each of the nq query rows xq[nq x d], the k nearest rows of
 * xr[nr x d] (Section 4.2, kNN = cdist + topk; exact as in Section 7's
 * exactness claim).
 *   idx_out[nq x k]  int64, reference row ids sorted by (distance, id)
 *   dist_out[nq x k] fp32, Euclidean distances (rounded from fp64)
 * opts may be NULL (defaults).  stats may be NULL.
 * Requires 1 <= k <= nr - exclude_self, k <= 256, d <= 4096.
 */
tod_status tod_knn(const float* xq, int64_t nq, const float* xr, int64_t nr, int64_t d,
                   int32_t k, const tod_options* opts, void* workspace, size_t ws_bytes,
                   void* stream, int64_t* idx_out, float* dist_out, tod_stats* stats);

/*
 * tod_knn for callers that cannot allocate device memory (serving loops that
 * keep allocation off their path, harnesses that forbid hipMalloc): the same
 * computation and outputs as tod_knn, with no workspace argument.  Its
 * workspace is a static device array of TOD_NOALLOC_SCRATCH_BYTES inside the
 * library, one per GPU (the loaded code object holds it until the process
 * ends); the call makes no hipMalloc, hipFree, HIP event or other allocating
 * call.  The planner fits the query blocks and reference splits into that
 * array as it does for a small caller workspace (tod_plan_workspace with
 * ws_bytes = TOD_NOALLOC_SCRATCH_BYTES gives the plan).
 *   TOD_ERR_WORKSPACE  the problem does not fit the array (not even one
 *                      32-row query block beside the fixed buffers, or
 *                      opts fixes query_block / ref_splits beyond it): use
 *                      tod_knn with a workspace of its own.
 * Every call on a GPU shares that GPU's array, and the array keeps the last
 * call's contents (each call initialises what it reads).  Calls that overlap
 * on one GPU (other threads, other streams) race on it: the caller
 * serialises them.  The call still synchronises `stream` before it returns,
 * so it cannot be captured into a HIP graph.  stats, if given, carries the
 * plan and row counts; its timings are 0 (no events are created).
 */
#define TOD_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
tod_status tod_knn_noalloc(const float* xq, int64_t nq, const float* xr, int64_t nr, int64_t d,
                           int32_t k, const tod_options* opts, void* stream, int64_t* idx_out,
                           float* dist_out, tod_stats* stats);

/*
 * kNN-OD scores of X against itself (each point's own row excluded), the
 * detector's fit (Appendix D's fit / decision_scores_):
 *   score_out[n] = opts->score of the k neighbour distances (default: the
 *                  distance to the k-th nearest neighbour, Table 1's kNN).
 * idx_out[n x k] and dist_out[n x k] are optional (NULL to skip).
 */
tod_status tod_knn_score(const float* x, int64_t n, int64_t d, int32_t k,
                         const tod_options* opts, void* workspace, size_t ws_bytes,
                         void* stream, float* score_out, int64_t* idx_out, float* dist_out,
                         tod_stats* stats);

/*
 * LOF of X against itself (Table 1; Breunig et al. 2000, exactly k
 * neighbours, self excluded):
 *   lof_out[n]       fp32 LOF scores (computed in fp64)
 *   knn_score_out[n] optional: kNN-OD score from the same neighbour lists
 *   idx_out, dist_out optional neighbour lists as in tod_knn
 * (The optional outputs cost no extra pass: LOF needs the exact lists and
 * k-distances anyway, so a caller that wants both detectors makes one call.)
 */
tod_status tod_lof(const float* x, int64_t n, int64_t d, int32_t k, const tod_options* opts,
                   void* workspace, size_t ws_bytes, void* stream, float* lof_out,
                   float* knn_score_out, int64_t* idx_out, float* dist_out, tod_stats* stats);

/*
 * LOF on Breunig et al.'s k-distance neighbourhoods (Table 1's LOF; a user
 * of neighbours within range, Section 5.3): every point tied at the
 * k-distance belongs, so a neighbourhood can hold more than k points.  For
 * every row p of X (its own row excluded):
 *   kd2(p)   = the k-th smallest D2(p, o), o != p
 *   N_k(p)   = {o != p : D2(p, o) <= kd2(p)}
 *   reach(p, o) = max(sqrt(kd2(o)), sqrt(D2(p, o)))
 *   lrd(p)   = 1 / (mean over N_k(p) of reach(p, o) + 1e-10)
 *   LOF(p)   = mean over N_k(p) of lrd(o), divided by lrd(p)
 * D2 is the fp64 squared distance summed over the columns in order without
 * fused multiply-adds; membership is decided exactly in it (as tod_nwr
 * decides range membership).  Where no distance ties the k-distance, N_k(p)
 * is the k nearest and the result is tod_lof's.
 * Steps: the exact kNN lists with k + 1 entries (as tod_knn, self excluded;
 * k entries when k = n - 1), kd2 from the first k; if every row's (k+1)-th
 * neighbour is farther than kd2 (by more than the summation orders can
 * differ), no point ties and the neighbourhoods are the k-lists; otherwise
 * they come from the range query at each row's own radius (tod_nwr's
 * fp16 / bf16 range filter with exact verification).  Then lrd and LOF.
 *   capacity         pairs (p, o) the workspace holds, summed over p; at
 *                    least n k (no ties)
 *   lof_out[n]       fp32 LOF scores (computed in fp64)
 *   count_out[n]     optional: |N_k(p)| (int32)
 * Workspace: tod_lof_ties_workspace_size(n, d, k, capacity, opts) bytes (0:
 * invalid sizes or options).  Requires d <= 512 and an fp16 / bf16 / AUTO
 * precision (TOD_ERR_UNSUPPORTED otherwise); opts->exclude_self is ignored
 * (always on).  TOD_ERR_CAPACITY if the neighbourhoods hold more than
 * capacity pairs: stats->pairs_in_range (when stats is given) then holds the
 * number needed, and lof_out is unspecified.
 */
size_t tod_lof_ties_workspace_size(int64_t n, int64_t d, int32_t k, int64_t capacity,
                                   const tod_options* opts);
tod_status tod_lof_ties(const float* x, int64_t n, int64_t d, int32_t k, int64_t capacity,
                        const tod_options* opts, void* workspace, size_t ws_bytes, void* stream,
                        float* lof_out, int32_t* count_out, tod_stats* stats);

/*
 * kNN-OD scores of new points xq[nq x d] against the fitted set xr[nr x d]
 * (Appendix D's decision_function, the inductive setting): the same score as
 * tod_knn_score, from the k nearest rows of xr, nothing excluded (a row of xr
 * passed again as a query is its own neighbour at distance 0).
 *   score_out[nq] fp32; idx_out, dist_out optional as in tod_knn.
 * opts->exclude_self must be 0.
 */
tod_status tod_knn_decision(const float* xq, int64_t nq, const float* xr, int64_t nr, int64_t d,
                            int32_t k, const tod_options* opts, void* workspace, size_t ws_bytes,
                            void* stream, float* score_out, int64_t* idx_out, float* dist_out,
                            tod_stats* stats);

/*
 * kNN classifier (Appendix B's kNN_CLF: cdist, topk, then a majority vote):
 * the predicted class of every row of xq is the most frequent label among
 * its k nearest rows of xr, ties going to the smallest label.
 *   labels_r[nr]  int32 (device), classes 0 .. n_classes - 1
 *   pred_out[nq]  int32 (device)
 * Requires 1 <= n_classes <= 65536 and opts->exclude_self == 0 (unless
 * xq == xr: then each point votes without itself).  A label outside
 * [0, n_classes) makes the call fail with TOD_ERR_INVALID_ARG (after the
 * kernels ran; pred_out is then unspecified).  Workspace: mode 2.
 */
tod_status tod_knn_classify(const float* xq, int64_t nq, const float* xr, int64_t nr, int64_t d,
                            int32_t k, const int32_t* labels_r, int32_t n_classes,
                            const tod_options* opts, void* workspace, size_t ws_bytes,
                            void* stream, int32_t* pred_out, tod_stats* stats);

/*
 * ABOD as Section 4.3 builds it from the kNN and cosine-similarity operators:
 * for every point of X (its own row excluded), the mean over the unordered
 * pairs {b, c} of its k nearest neighbours of the cosine of the angle between
 * x_b - x_i and x_c - x_i (fp64, rounded to fp32).  Pairs with a
 * zero-length difference (a duplicate of x_i) are left out; a point without
 * any pair left scores 0.  Higher means more outlying (the neighbours lie in
 * one direction).
 *   score_out[n] fp32; idx_out, dist_out optional lists as in tod_knn.
 * Requires 2 <= k <= 64 (TOD_ERR_INVALID_ARG below, TOD_ERR_UNSUPPORTED above).
 * Workspace: mode 1 of tod_workspace_size.
 */
tod_status tod_abod(const float* x, int64_t n, int64_t d, int32_t k, const tod_options* opts,
                    void* workspace, size_t ws_bytes, void* stream, float* score_out,
                    int64_t* idx_out, float* dist_out, tod_stats* stats);

/*
 * COF, the connectivity-based outlier factor (Tang et al.; Table 1), of
 * every point of X (its own row excluded).  For point p and G = {p} plus its
 * k nearest neighbours, the set-based nearest path starts from {p} and adds,
 * k times, the point of G nearest to the points added so far (distance to a
 * set = smallest distance to a member; ties to the lower row index); step i
 * costs that distance c_i.  The average chaining distance is
 *   ac(p) = sum_i 2 (k + 1 - i) / (k (k + 1)) c_i
 * and COF(p) = (ac(p) + 1e-10) / (mean over the neighbours o of ac(o) + 1e-10)
 * (fp64, rounded to fp32; the 1e-10 keeps duplicates finite, as LOF's does).
 *   cof_out[n] fp32; knn_score_out, idx_out, dist_out optional as in tod_lof.
 * Requires 1 <= k <= 63 (TOD_ERR_UNSUPPORTED above).  Workspace: mode 1.
 */
tod_status tod_cof(const float* x, int64_t n, int64_t d, int32_t k, const tod_options* opts,
                   void* workspace, size_t ws_bytes, void* stream, float* cof_out,
                   float* knn_score_out, int64_t* idx_out, float* dist_out, tod_stats* stats);

/*
 * Host-only planner (Section 6 automatic batching): fills *plan with the
 * precision, K', query block, reference splits and block count that tod_knn
 * would use, without touching the GPU.  Only the plan fields of tod_stats
 * are written; tile_launches counts one launch per block (the tail split is
 * decided at run time from the GPU's occupancy).
 */
tod_status tod_plan(int64_t nq, int64_t nr, int64_t d, int32_t k, const tod_options* opts,
                    tod_stats* plan);

/*
 * The plan a call would use with a workspace of ws_bytes (Section 6:
 * automatic batching sized to the memory at hand; the paper batches so that
 * large inputs fit a GPU's memory).  A workspace smaller than
 * tod_workspace_size() is not an error by itself: the query block shrinks to
 * what the room beside the fixed buffers (quantised copies, norms, radii,
 * worklist, neighbour lists) holds, at S x K' x 8 bytes per query row, the
 * reference splits S follow the smaller block, and the rows run in more
 * blocks with identical results.  TOD_ERR_WORKSPACE if not even one 32-row
 * block fits, or if opts fixes query_block or ref_splits and the plan does
 * not fit.  mode as in tod_workspace_size; the plan is for X against itself
 * when mode == 1 or opts->exclude_self is set, else for separate sets.
 * Host only, like tod_plan.
 */
tod_status tod_plan_workspace(int64_t nq, int64_t nr, int64_t d, int32_t k, int32_t mode,
                              const tod_options* opts, size_t ws_bytes, tod_stats* plan);

/*
 * Neighbours within range (NWR, Section 5.3: the case study of provable
 * quantization).  For every query row i, the reference rows j whose
 * Euclidean distance is at most phi.  The decision is exact: a pair is in
 * range iff its squared distance, summed in fp64 over the columns in order
 * from the fp32 rows ((double)x - (double)y, squared, added), is at most
 * phi * phi rounded to fp64.  The filter evaluates every pair in fp16 / bf16
 * (MFMA, fp32 accumulation); pairs it can place on neither side of phi with
 * certainty (Eq. (nwr-check)'s test |D - phi| > Err, with this library's
 * error bound) are recomputed exactly, the others are decided by the filter.
 *   row_ptr_out[nq + 1] int64 (device): CSR offsets, row i's pairs occupy
 *                       [row_ptr_out[i], row_ptr_out[i + 1]).  Always written.
 *   idx_out[capacity]   int64 (device), nullable: reference ids, ascending
 *                       within a row.  NULL = count only.
 *   dist_out[capacity]  fp32 (device), nullable: their Euclidean distances
 *                       (fp64 rounded to fp32).
 *   total_out           HOST pointer, nullable: the number of pairs in range.
 * opts: precision AUTO (= FP16) or FP16 / BF16 (FP32 is TOD_ERR_UNSUPPORTED:
 * the range filter is an MFMA tile), exclude_self (drops j == i; requires
 * xq == xr and nq == nr), ref_splits, margin_scale, force_fallback (no pair
 * is ruled in by the filter: every candidate is recomputed).  shortlist,
 * query_block, no_recheck and reorder do not apply.
 * Workspace: a fixed part plus room for candidate pairs (8 bytes each);
 * tod_nwr_workspace_size() gives the fixed part plus room for 64 candidates
 * per query row and 2^20 more.  Any extra bytes are used as candidate room.
 * Query rows are processed in as many batches (of multiples of 32 rows) as
 * that room needs: automatic batching sized to memory (Section 6).
 * TOD_ERR_WORKSPACE if 32 consecutive query rows have more candidates than
 * the room holds (tod_last_error() names the bytes needed).
 * TOD_ERR_CAPACITY if idx_out is given and the total exceeds capacity; then
 * row_ptr_out and *total_out are valid and idx_out / dist_out unspecified.
 * Requires phi finite and >= 0, d <= 512.
 */
size_t tod_nwr_workspace_size(int64_t nq, int64_t nr, int64_t d, const tod_options* opts);
tod_status tod_nwr(const float* xq, int64_t nq, const float* xr, int64_t nr, int64_t d,
                   double phi, const tod_options* opts, void* workspace, size_t ws_bytes,
                   void* stream, int64_t* row_ptr_out, int64_t capacity, int64_t* idx_out,
                   float* dist_out, int64_t* total_out, tod_stats* stats);

/*
 * LOCI, the multi-granularity deviation factor of Papadimitriou et al.
 * (one of Table 1's proximity-based detectors; like LOF it is built on
 * neighbours within range, Section 5.3), at a ladder of sampling radii
 * r_0 < r_1 < ... < r_{L-1}.  For every row p of X and every radius r_l:
 *   n_alpha[p][l] = |{q : d(p, q) <= alpha r_l}|  (counting neighbourhood)
 *   n_r[p][l]     = |{q : d(p, q) <= r_l}|        (sampling neighbourhood)
 * (p itself belongs to both); n_hat and sigma are the mean and the population
 * standard deviation of n_alpha[q][l] over q in the sampling neighbourhood,
 *   MDEF = 1 - n_alpha[p][l] / n_hat,   sigma_MDEF = sigma / n_hat.
 * Membership is exact, as in tod_nwr: d(p, q) <= r iff the fp64 squared
 * distance summed over the columns in order is <= fl(r * r), and
 * d(p, q) <= alpha r iff it is <= fl(fl(alpha * r)^2).  The neighbourhood
 * sums S1 = sum n_alpha[q][l] and S2 = sum n_alpha[q][l]^2 are exact 64-bit
 * integers; then, in fp64 and in this order, n_hat = S1 / n_r,
 * var = S2 / n_r - n_hat * n_hat (negative values become 0),
 * sigma = sqrt(var), MDEF, sigma_MDEF.  A radius counts for p when
 * n_r[p][l] >= n_min.  flag_out[p] = 1 when MDEF > k_sigma * sigma_MDEF at a
 * counted radius; score_out[p] = the largest MDEF / sigma_MDEF over the
 * counted radii, where a radius with sigma_MDEF = 0 (all samples equal, so
 * MDEF = 0) contributes 0, and 0 when no radius counts.
 *   radii               HOST array [n_radii] fp64, strictly increasing, >= 0,
 *                       finite; 1 <= n_radii <= 32.
 *   alpha               in (0, 1]; n_min >= 1; k_sigma finite, >= 0.
 *   capacity            pairs (p, q) with d(p, q) <= r_{L-1}, self pairs
 *                       included, that the workspace holds.  If more are in
 *                       range the call returns TOD_ERR_CAPACITY and, when
 *                       stats is given, stats->pairs_in_range = the number
 *                       needed (size the workspace for it and call again).
 *   score_out[n]        fp64 (device).
 *   flag_out[n]         int32 (device), nullable.
 *   n_alpha_out, n_r_out [n * n_radii] int32 (device), nullable, row-major
 *                       (radius fastest).
 *   mdef_out, sigma_mdef_out [n * n_radii] fp64 (device), nullable.
 * opts as tod_nwr (precision AUTO / FP16 / BF16, ref_splits, margin_scale,
 * force_fallback); exclude_self must be 0 (p samples itself).  Requires
 * n <= 2^20, which keeps S2 below 2^63 (TOD_ERR_UNSUPPORTED above).
 * Workspace: tod_loci_workspace_size(n, d, n_radii, capacity, opts) bytes,
 * 256-byte aligned; stats: the neighbours-within-range pass's fields, with
 * ms_score the time of the two LOCI kernels.
 */
size_t tod_loci_workspace_size(int64_t n, int64_t d, int32_t n_radii, int64_t capacity,
                               const tod_options* opts);
tod_status tod_loci(const float* x, int64_t n, int64_t d, const double* radii, int32_t n_radii,
                    double alpha, int32_t n_min, double k_sigma, int64_t capacity,
                    const tod_options* opts, void* workspace, size_t ws_bytes, void* stream,
                    double* score_out, int32_t* flag_out, int32_t* n_alpha_out,
                    int32_t* n_r_out, double* mdef_out, double* sigma_mdef_out,
                    tod_stats* stats);

/*
 * Sequence operators: rows for the detectors from token sequences.
 *
 * The rows that outlier detectors score are often a language model's hidden
 * states.  These operators are what such a model needs beside its matrix
 * products: attention over packed prompts, and a paged cache of keys and
 * values with attention of each sequence's newest tokens over it.
 *
 * They differ from the calls above in three ways: tensors are fp16 or bf16
 * (TOD_PREC_FP16, TOD_PREC_BF16); lengths, tables and slots are read on the
 * device; and a call returns once its work is queued on `stream`, without
 * waiting and without allocating, so that it may be captured into a HIP graph.
 * The status therefore covers the arguments and the launch, not the values
 * that lengths and tables hold: those never lead outside the buffers whose
 * sizes are given, whatever they are, and each operator says what becomes of
 * values out of range.  All buffers stay untouched by others until the work is
 * done.  tod_last_error() works as for the calls above.
 *
 * Packed sequences: n_seq sequences share `tokens` rows; sequence s holds the
 * rows row_start[s] .. row_start[s + 1] - 1 (int32 [n_seq + 1], ascending from
 * 0; entries are cut to [0, tokens]).  Sequences may be empty.  Where starts do
 * not ascend, the call's output rows are unspecified and may stay unwritten.
 *
 * Paged cache: k_pages and v_pages are [n_pages, kv_heads, page_rows, dim],
 * contiguous.  table[n_seq, table_cols] (int32) holds a sequence's pages in
 * order: the token at position p lies in page table[s][p / page_rows], row
 * p % page_rows; its slot is page * page_rows + row.
 */

/*
 * Map of the cache for a step: pages and slots of every sequence's new tokens.
 * cached[s] tokens of sequence s lie in the cache and fresh[s] follow (int32;
 * negative counts as 0).  With P = page_rows and C = table_cols,
 *   have(s) = min(ceil(cached / P), C)
 *   need(s) = min(ceil((cached + fresh) / P), C) - have(s)
 * The pages needed, over the sequences in order, take free_pages[0 .. n_free)
 * from its start, -1 where it ends; table[s][have .. have + need) receives
 * them, other entries stay.  The call may be repeated on its own result.
 *   row_start_out[n_seq + 1] int32: packed rows of the new tokens
 *   slot_out[tokens] int64: the slot of every new token; -1 where it has no
 *                    page, its position lies past the table, or the row past
 *                    the last sequence
 *   pos_out[tokens]  int32, nullable: its position (cached + its number), or
 *                    -1 for rows past the last sequence
 *   used_out[2]      int64, nullable: pages needed, and new tokens left
 *                    without a slot (free_pages at its end, the table at its
 *                    last column or without the page that was begun, or more
 *                    new tokens than `tokens`: those are left out and need no
 *                    pages).  Entries of free_pages are page ids >= 0.
 */
tod_status tod_page_map(const int32_t* cached, const int32_t* fresh, int64_t n_seq,
                        const int32_t* free_pages, int64_t n_free, int32_t page_rows,
                        int32_t* table, int64_t table_cols, int64_t tokens, void* stream,
                        int32_t* row_start_out, int64_t* slot_out, int32_t* pos_out,
                        int64_t* used_out);

/*
 * Write of new keys and values into their slots (16-bit elements of any type,
 * moved unchanged).  k, v: [tokens, kv_heads, dim], elements of a row
 * contiguous; *_row and *_head are the strides of tokens and heads in elements,
 * multiples of 8 (0: contiguous).  A token whose slot is outside
 * [0, n_pages * page_rows) is left out; a slot that several tokens share ends
 * up with pieces of any of them.  dim is a multiple of 8; tensors are 16-byte aligned.
 */
tod_status tod_page_write(const void* k, const void* v, int64_t tokens, int32_t kv_heads,
                          int32_t dim, int64_t k_row, int64_t k_head, int64_t v_row,
                          int64_t v_head, const int64_t* slot, void* k_pages, void* v_pages,
                          int64_t n_pages, int32_t page_rows, void* stream);

/* Heads, types and strides of an attention call. */
typedef struct {
  uint32_t struct_size; /* must be sizeof(tod_attn) */
  int32_t precision;    /* of q, k, v and out: TOD_PREC_FP16 or TOD_PREC_BF16 */
  int32_t heads;        /* query heads */
  int32_t kv_heads;     /* key / value heads; query head h reads head h / (heads / kv_heads) */
  int32_t dim;          /* elements of a head: a multiple of 8, at most 256 */
  int32_t causal;       /* 1: a token sees itself and those before it; 0 (tod_attn_prompt only):
                         * all of its sequence */
  float scale;          /* of q k^T, finite, > 0; 0: 1 / sqrt(dim) */
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;
                        /* strides of tokens and heads in elements, multiples of 8; 0: those of a
                         * contiguous [tokens, heads, dim].  The elements of a head are
                         * contiguous.  k_* and v_*: tod_attn_prompt only. */
} tod_attn;

void tod_default_attn(tod_attn* attn, int32_t heads, int32_t kv_heads, int32_t dim,
                      int32_t precision);

/*
 * Attention over whole packed prompts.  For query head h of token i, over the
 * tokens j of the same sequence that i sees:
 *   s_j = scale <q_i, k_j>,  out_i = sum_j exp(s_j) v_j / sum_j exp(s_j),
 *   lse_i = ln sum_j exp(s_j)
 * in one pass with fp32 products, maxima, sums and accumulators (the weights
 * are rounded to the input type for their product with v).
 *   q [tokens, heads, dim], k, v [tokens, kv_heads, dim]; 16-byte aligned
 *   out [tokens, heads, dim] contiguous; lse_out [tokens, heads] fp32, nullable
 * A row that sees no key, such as one past row_start[n_seq], gets 0 and -inf.
 * Keys and values that a row does not see do not reach it, whatever they hold.
 * Where it sees values that are infinite or NaN, their sum is its output in
 * that column (every weight counts as positive, however small); a NaN score
 * makes the row NaN.
 * Workspace: tod_attn_workspace_size(attn, tokens, n_seq, tokens) bytes, 256-byte
 * aligned (0: invalid sizes); nothing in it lasts beyond the call.
 */
size_t tod_attn_workspace_size(const tod_attn* attn, int64_t tokens, int64_t n_seq,
                               int64_t max_fresh);
tod_status tod_attn_prompt(const tod_attn* attn, const void* q, const void* k, const void* v,
                           int64_t tokens, const int32_t* row_start, int64_t n_seq,
                           void* workspace, size_t ws_bytes, void* stream, void* out,
                           float* lse_out);

/*
 * Attention of every sequence's new tokens over its pages: chunks of a prompt,
 * single tokens, or both.  Sequence s has cached[s] tokens in the cache before
 * this step, and its rows of q are the tokens that follow, whose keys and
 * values have been written too: token i of them sees the positions
 * 0 .. cached[s] + i (at most table_cols * page_rows of them, which with the
 * tokens and 64 stay below 2^31).  Formulas and outputs
 * as tod_attn_prompt; attn->causal must be 1.  An entry of the table that is
 * no page counts as a page of zeros.
 *   max_fresh  no sequence has more new tokens than this (tokens is always
 *              right).  Rows of a sequence that has are unspecified.
 * Workspace: tod_attn_workspace_size(attn, tokens, n_seq, max_fresh) bytes,
 * 256-byte aligned (0: invalid sizes); nothing in it lasts beyond the call.
 */
tod_status tod_attn_paged(const tod_attn* attn, const void* q, const void* k_pages,
                          const void* v_pages, int64_t n_pages, int32_t page_rows,
                          const int32_t* table, int64_t table_cols, const int32_t* row_start,
                          const int32_t* cached, int64_t n_seq, int64_t tokens,
                          int64_t max_fresh, void* workspace, size_t ws_bytes, void* stream,
                          void* out, float* lse_out);

/*
 * Appends: a step's new keys and values into the cache with the position
 * rotation applied on the way, and the rotated queries.  Of the first `rotary`
 * = r elements of a head, the pairs (x_i, x_{i + r/2}), or with `interleaved`
 * (x_2i, x_2i+1), i < r / 2, turn by the angle t = pos * rates[i]:
 *   (x, y) -> (x cos t - y sin t, x sin t + y cos t)
 * The angle is formed and reduced to a quarter turn in 64 bits, and with what the
 * product of position and rate loses past them, however far the position.  Values
 * and the elements from r on are not rotated.
 */
typedef struct {
  uint32_t struct_size; /* must be sizeof(tod_append) */
  int32_t precision;    /* of q, k, v and q_out: TOD_PREC_FP16 or TOD_PREC_BF16 */
  int32_t heads;        /* query heads */
  int32_t kv_heads;     /* key / value heads */
  int32_t dim;          /* elements of a head: a multiple of 8, at most 256 */
  int32_t rotary;       /* rotated elements of a head: even, at most dim; 0: none */
  int32_t interleaved;  /* 1: pairs of neighbours; 0: pairs rotary / 2 apart */
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;
                        /* strides as in tod_attn */
} tod_append;

void tod_default_append(tod_append* append, int32_t heads, int32_t kv_heads, int32_t dim,
                        int32_t precision);

/*
 * Append to a paged cache of 16-bit rows.
 *   q [tokens, heads, dim], k, v [tokens, kv_heads, dim]; 16-byte aligned
 *   pos[tokens] int32: positions, as of tod_page_map (any sign: a row of q whose
 *                 token has no slot is rotated as every other)
 *   rates[rotary / 2] fp32 (device): angle of a step of one position; NULL if
 *                 rotary is 0
 *   slot, k_pages, v_pages: as in tod_page_write
 *   q_out [tokens, heads, dim] contiguous, sharing no memory with q, k or v
 * Rotated elements are fp32 sums of two products with an fp32 cosine and sine, then
 * rounded to the type.  Of a slot that several tokens share, parts of the row may come
 * from different ones.
 */
tod_status tod_page_append(const tod_append* append, const void* q, const void* k, const void* v,
                           int64_t tokens, const int32_t* pos, const float* rates,
                           const int64_t* slot, void* k_pages, void* v_pages, int64_t n_pages,
                           int32_t page_rows, void* stream, void* q_out);

/*
 * A paged cache of 4-bit rows: 4.25 bits an element.  A row's elements come in
 * blocks of 32.  Element i of a row is the code in byte i / 2 of the row, its low
 * half where i is even: codes 0 .. 7 stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6, and
 * 8 + c for the negative of c.  Byte b of a block scales them by 2^(b - 127);
 * with 255 all of them are NaN.  An operator takes the values as numbers of its
 * tensors' type (beyond its largest: infinite).
 * dim is a multiple of 32; table and slots are as over 16-bit pages.
 */
typedef struct {
  uint32_t struct_size; /* must be sizeof(tod_cache4) */
  int32_t page_rows;
  int64_t n_pages;
  void *k_codes, *v_codes;       /* [n_pages, kv_heads, page_rows, dim / 2] */
  uint8_t *k_scales, *v_scales;  /* [n_pages, kv_heads, page_rows, dim / 32] */
                                 /* all four 16-byte aligned */
} tod_cache4;

/*
 * Append to a 4-bit cache; arguments as in tod_page_append.  For a block whose
 * largest magnitude is a, the scale is the smallest 2^e with a <= 7 2^e, e cut to
 * [-23, 13] for fp16 and to [-125, 125] for bf16 (so that every value is one of
 * the type); each element over 2^e is rounded to the nearest value, ties to
 * the even code, beyond 6 to 6.  A block that holds an infinity or a NaN gets the byte 255
 * and the codes 0.  Rotated keys are scaled and rounded in 64 bits, without a
 * rounding to 16 bits before.  Of a slot that several tokens share, codes and
 * scales may come from different ones.
 */
tod_status tod_page_append4(const tod_append* append, const void* q, const void* k, const void* v,
                            int64_t tokens, const int32_t* pos, const float* rates,
                            const int64_t* slot, const tod_cache4* cache, void* stream,
                            void* q_out);

/*
 * Rows of a 4-bit cache as 16-bit elements: k_out, v_out [tokens, kv_heads, dim],
 * contiguous and 16-byte aligned.  Tokens whose slot is outside the cache get zeros.
 */
tod_status tod_page_read4(const tod_cache4* cache, int32_t kv_heads, int32_t dim,
                          int32_t precision, const int64_t* slot, int64_t tokens, void* stream,
                          void* k_out, void* v_out);

/*
 * tod_attn_paged over a 4-bit cache: the same formulas, over the values that the
 * codes stand for, and the same outputs and rules.  attn->dim is a multiple
 * of 32; attn->precision is that of q and out.
 * Workspace: tod_attn_paged4_workspace_size(attn, tokens, n_seq, max_fresh) bytes,
 * 256-byte aligned (0: invalid sizes); nothing in it lasts beyond the call.
 */
size_t tod_attn_paged4_workspace_size(const tod_attn* attn, int64_t tokens, int64_t n_seq,
                                      int64_t max_fresh);
tod_status tod_attn_paged4(const tod_attn* attn, const void* q, const tod_cache4* cache,
                           const int32_t* table, int64_t table_cols, const int32_t* row_start,
                           const int32_t* cached, int64_t n_seq, int64_t tokens,
                           int64_t max_fresh, void* workspace, size_t ws_bytes, void* stream,
                           void* out, float* lse_out);

/* Static string naming a status code. */
const char* tod_status_string(tod_status status);

/* Detail of the last error on the calling thread ("" if none). */
const char* tod_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* TOD_H */
