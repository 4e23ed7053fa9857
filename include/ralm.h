/*
 * ralm.h — C ABI of the MI355X (gfx950) retrieval hot path of RaLMSpec
 * (arXiv 2401.14021, "Accelerating Retrieval-augmented Language Model Serving
 * with Speculation").
 *
 * Four operations of the paper's serving loop (Alg. 1) are implemented:
 *
 *   C.retrieve(q_1..q_s)   batched exact knowledge-base retrieval, the
 *                          verification step        -> ralm_retrieve_topk[_ex]
 *   Q.retrieve(q_i)        speculative retrieval from the request's local
 *                          cache, top-1             -> ralm_cache_lookup
 *   m = argmin_i d^_i!=d_i first mis-speculated step -> ralm_verify
 *   Q.insert(C.retrieve(..)) cache update after verification -> ralm_cache_insert
 *
 * and, around that loop: the stride scheduler of Section 4 as host functions
 * (ralm_os3_*), and for KNN-LM datastores (Section 5.3) ranking by distance
 * (RALM_METRIC_L2) and the neighbour distribution (ralm_knnlm_probs).
 *
 * For the generator that runs next to the loop, on the card that the datastore
 * shares: a paged cache of keys and values in 4 bits, attention over it, the
 * forking, rolling back and compacting of its pages (ralm_kv_*), and the
 * verification of drafted tokens against a target's probabilities
 * (ralm_verify_draft).  Around that attention: products with their epilogues
 * (ralm_linear), norms of the residual stream (ralm_residual_norm), rotary
 * positions on the way into the cache (ralm_kv_append_rotary), and the mixture
 * of the model's and the neighbours' distributions (ralm_knnlm_target).
 *
 * General conventions
 *   - Unless a parameter says "host", every data pointer is a DEVICE pointer
 *     owned by the caller.  The library keeps no reference after the call's
 *     work has run and never frees caller memory.
 *   - Calls enqueue work on the given HIP stream (a hipStream_t passed as
 *     void*; NULL = the default stream) and return without synchronising,
 *     except where stated.  Work of one call is ordered on that stream.
 *     Apart from ralm_retrieve_topk, ralm_workspace_overflows and
 *     ralm_workspace_counters, a call only
 *     launches kernels (no allocation, no memset or copy nodes), so after one
 *     ordinary call of the same shapes (the first launch of a kernel sets its
 *     attributes) it may be recorded into a HIP graph and replayed.
 *   - Matrices are row-major.  ids are int32 row numbers of the datastore
 *     (N <= 2^31 - 512); sizes are int64.  A call takes at most 2^20 queries
 *     and 2^22 requests (RALM_ERR_SHAPE beyond that).
 *   - The ranking is always (score descending, row id ascending): equal scores
 *     go to the lower id.  The paper does not define ties; this is this
 *     library's rule, at every stage.
 *   - The score is the inner product, or minus the squared distance (see
 *     ralm_metric).  Final scores (outputs) are the fp32 rounding of a sum
 *     formed in double from fp32 (or exactly widened fp16/bf16) inputs.
 *   - Argument errors are detected on the host before anything is launched and
 *     are reported as a status; ralm_last_error() gives the text.  Inputs are
 *     assumed finite (NaN/Inf: behaviour unspecified) where nothing else is said.
 */
#ifndef RALM_H
#define RALM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RALM_OK = 0,
    RALM_ERR_NULL = 1,      /* a required pointer is NULL */
    RALM_ERR_SHAPE = 2,     /* Q, N, d, R, C or a stride is out of range */
    RALM_ERR_K = 3,         /* k < 1, k > N, k > RALM_MAX_K, k' < k or k' > RALM_MAX_K_PRIME */
    RALM_ERR_DTYPE = 4,     /* dtype tag unknown or not allowed in that slot */
    RALM_ERR_ALIGN = 5,     /* base pointer or row pitch not 16-byte aligned */
    RALM_ERR_WORKSPACE = 6, /* workspace NULL, misaligned or too small */
    RALM_ERR_RANGE = 7,     /* a count (Qt, true_stride) is negative or does not fit */
    RALM_ERR_DEVICE = 8,    /* a HIP call failed (text in ralm_last_error) */
    RALM_ERR_OVERFLOW = 9   /* a candidate buffer overflowed (degenerate input); see below */
} ralm_status;

typedef enum { RALM_F32 = 0, RALM_BF16 = 1, RALM_F16 = 2 } ralm_dtype;

/*
 * Score of a row x for a query q.  RALM_METRIC_IP: the inner product <q, x>
 * (dense passage retrieval).  RALM_METRIC_L2: minus the squared Euclidean
 * distance, -|q - x|^2 (KNN-LM datastores rank their entries by distance,
 * Section 5.3), so that a larger score is a better match under both.
 */
typedef enum { RALM_METRIC_IP = 0, RALM_METRIC_L2 = 1 } ralm_metric;

#define RALM_MAX_K 1024
#define RALM_MAX_K_PRIME 4096

/*
 * The knowledge base as the flat index of an exact dense retriever
 * (Section 5.1, "Retrievers"): N key vectors of dimension d.
 *
 *   exact  the keys that define the right answer: fp32 [N, d], or fp16 [N, d]
 *          (KNN-LM keys; widened exactly).  Scores returned to the caller are
 *          computed from this copy.
 *   scan   the copy the full scan reads: bf16 or fp16 roundings of the exact
 *          keys (build with ralm_build_scan_copy), or the exact copy itself
 *          (fp32 is rounded to bf16 on the fly: at or near the HBM rate for
 *          batches of up to 256 queries, at about half the speed of a bf16
 *          copy for larger ones; fp16 is used as is).
 *          NULL means "use the exact copy".
 *   *_stride  row pitch in ELEMENTS (0 = d).  Pitch in bytes and both base
 *          pointers must be multiples of 16.  d must be a multiple of 8.
 *   metric RALM_METRIC_IP (0) or RALM_METRIC_L2.  With RALM_METRIC_L2 the scan
 *          copy is mandatory, bf16 or fp16, and its rows have d + 8 columns:
 *          the d rounded elements, then the row's squared norm as the sum of
 *          two scan-dtype numbers, then six zeros (ralm_build_scan_copy_l2
 *          writes this layout; scan_stride 0 = d + 8, but a pitch that is a
 *          multiple of 64 elements keeps rows on 128-byte lines and scans
 *          ~20 % faster).  The scan then scores a
 *          row as 2<q, x> - |x|^2 on the matrix cores with no change to its
 *          kernels; final scores are -|q - x|^2 from the exact copy.
 */
typedef struct {
    const void *exact;
    int32_t exact_dtype;    /* RALM_F32 or RALM_F16 */
    const void *scan;       /* may be NULL */
    int32_t scan_dtype;     /* RALM_BF16, RALM_F16 or RALM_F32 */
    int64_t N;
    int32_t d;
    int64_t exact_stride;
    int64_t scan_stride;
    int32_t metric;         /* RALM_METRIC_IP or RALM_METRIC_L2 */
} ralm_datastore_t;

/*
 * Batched exact retrieval, simplest form (Alg. 1, the batched verification
 * step; exact dense retriever of Section 5.1).
 *
 *   queries    device fp32 [Q, d]
 *   datastore  device fp32 [N, d]; it is both the exact and the scanned copy
 *   out_ids    device int32 [Q, k]; out_scores device fp32 [Q, k]; each row
 *              ranked best first.
 *
 * Runs on the default stream and synchronises before returning.  It uses
 * buffers of its own, kept between calls and grown on demand (allocating tens
 * of gigabytes per call is slow); ralm_release_buffers() frees them: the
 * workspace and, for batches of more than 768 queries only, a bf16 copy of the
 * datastore for the scan (N*d*2 bytes, rebuilt on every call; skipped if the
 * device has no room for it).  Batches of up to 768 queries scan the fp32 rows
 * as they are (21M x 768: about 9.3 ms for up to 64 queries, the rate at which
 * HBM delivers the rows; 14 ms for 256, 25 ms for 512), and hold no copy.  Calls are serialised.  Meant for convenience; a caller that
 * retrieves large batches repeatedly keeps a scan copy and uses the full form.
 * A query that the full form would leave unanswered (see
 * ralm_retrieve_topk_ex) makes the call retry through ralm_retrieve_topk_seq;
 * if it is still unanswered the call returns RALM_ERR_OVERFLOW.
 */
ralm_status ralm_retrieve_topk(const float *queries, int64_t Q, const float *datastore, int64_t N,
                               int32_t d, int32_t k, int32_t *out_ids, float *out_scores);

/* Frees the device buffers, and the word of pinned host memory, that ralm_retrieve_topk keeps between calls (synchronises). */
void ralm_release_buffers(void);

/* Bytes of workspace ralm_retrieve_topk_ex needs for (Q, ds, k, k_prime); 0 on bad arguments. */
size_t ralm_workspace_bytes(int64_t Q, const ralm_datastore_t *ds, int32_t k, int32_t k_prime);

/*
 * Batched exact retrieval, full form.  How it gets the exact answer from a
 * low-precision scan: every row is scored in the scan dtype on the matrix
 * cores with fp32 accumulation; per query the k' (>= k) best scan scores are
 * kept; those k' rows are re-scored from the exact copy and the best k of them
 * are returned.  k_prime = 0 picks a default (64 for k <= 32, else the power
 * of two >= 2k).
 *
 * That answer is the exact one unless the scan's rounding pushed a true top-k
 * row out of the k' kept ones.  The library checks this per query, on the
 * device: the margin (see out_margin) must exceed 8x the root mean square of
 * the differences between scan score and exact score seen on the query's own k'
 * candidates (when all of those differences are zero, a margin of zero is
 * enough).  A query that fails the check, or whose candidate list lost entries
 * (below), is answered again in the same call by an exact pass: every row of
 * the exact copy is scored exactly (the arithmetic of the final scores) and the
 * best k of the rows that reach the exact rank-k score found so far are
 * returned, which is the exact top k by construction.  The pass is skipped
 * when no query needs it; it reads the exact copy once per 16 such queries
 * (inner product on the fp64 matrix cores; 21M x 768 fp32: about 11 ms per
 * pass), once per 8 for the squared distance and for row lengths that are not
 * a multiple of 64 (fp32) or 128 (fp16) elements (13 to 26 ms).  With k_prime = k there is
 * no margin to speak of and nearly every query takes that pass.
 * ralm_workspace_counters reports how many did.
 *
 *   queries     device fp32 [Q, d] (host code never reads it)
 *   ds          HOST struct of device pointers
 *   out_ids / out_scores  device [Q, k] as above
 *   out_margin  optional device fp32 [Q] (may be NULL): exact score of the
 *               rank-k row among the candidates minus the scan score of the
 *               k'-th kept candidate (brought to the same scale under
 *               RALM_METRIC_L2), or minus the score that the last rows had to
 *               reach to be admitted where that is higher (below).  A row outside the candidates can belong in
 *               the top k only if the scan mis-scored it by at least this
 *               much.  Diagnostic: the library acts on it by itself (above).
 *               +inf when every row was a candidate (N < k').
 *   workspace   device scratch, 256-byte aligned, >= ralm_workspace_bytes();
 *               contents are undefined between calls; two calls that overlap
 *               in time must not share it.
 *   stream      hipStream_t
 *
 * The rows are visited in a fixed strided order, coarse samples first, and a
 * query's candidate list (a fixed number of slots in the workspace) takes only
 * scores that beat a score of the rows visited before: the one of the rank that
 * the final k'-th best is expected to have in that sample, five standard
 * deviations and a little more below, never better than a quarter of the way
 * from rank k to rank k', and never nearer to the score of rank k than what
 * rounding can do to a score (then it is the k'-th best).  If the order of the rows has it that fewer than k'
 * rows beat it in the end, the check's margin is taken from it.  Does not
 * synchronise.  If the list of some query overflows (only when the order of
 * the rows is correlated with that stride pattern, e.g. every other 256-row
 * tile holding the best matches), the list keeps what it has, the scan goes
 * on, and the query is answered by the exact pass, whose list holds only rows
 * that reach the exact rank-k score of the candidates that survived.  Only if
 * that list overflows too (more rows than it has slots, at least 16384, beat that score, tie with it,
 * or fall short of it by no more than one fp32 step: the pass forms its double
 * sums in another order than the re-score and leaves that much room)
 * are the query's outputs set to id -1 / score NaN; ralm_workspace_overflows()
 * counts those.  (Such a datastore holds tens of thousands of rows that no
 * fp32 score separates from the query's k-th best; a larger k would be the
 * honest request.)
 */
ralm_status ralm_retrieve_topk_ex(const float *queries, int64_t Q, const ralm_datastore_t *ds,
                                  int32_t k, int32_t k_prime, int32_t *out_ids, float *out_scores,
                                  float *out_margin, void *workspace, size_t workspace_bytes,
                                  void *stream);

/*
 * Same arguments, same result as ralm_retrieve_topk_ex, computed block by
 * block over consecutive rows: every block is small enough that a list holds
 * its k' best so far plus every row of the block, so no list can overflow
 * whatever the order of the rows.  About N / 16000 small launches instead of a
 * dozen large ones (21M rows: ~50 ms); meant as the retry after an overflow.
 */
ralm_status ralm_retrieve_topk_seq(const float *queries, int64_t Q, const ralm_datastore_t *ds,
                                   int32_t k, int32_t k_prime, int32_t *out_ids, float *out_scores,
                                   float *out_margin, void *workspace, size_t workspace_bytes,
                                   void *stream);

/*
 * Number of queries of the LAST ralm_retrieve_topk_ex / _seq call on this workspace
 * that were left unanswered (id -1 / score NaN).  Synchronises `stream` and
 * copies one int to the host (*count is a host pointer).
 */
ralm_status ralm_workspace_overflows(const void *workspace, void *stream, int32_t *count);

/*
 * Counters of the LAST ralm_retrieve_topk_ex / _seq call on this workspace, all
 * numbers of queries (host struct; synchronises `stream`).  All zero, as are
 * the other reports, for a workspace that holds no call's:
 *   unanswered        id -1 / score NaN (what ralm_workspace_overflows returns)
 *   ladder_overflows  candidate list lost entries during the scan; answered by
 *                     the exact pass
 *   hard_certified    margin above the deterministic bound of the scan's
 *                     rounding, (u_q + u_x + u_q u_x) |q| |x| + d 2^-24 |q| |x|
 *                     with unit roundoffs u = 2^-8 (bf16) or 2^-11 (fp16) of the
 *                     query and of the rows (0 for rows scanned as they are) and
 *                     |x| the longest of the query's candidates: a proof when
 *                     no row is longer than that, e.g. for unit-norm rows
 *   soft_certified    passed the check described at ralm_retrieve_topk_ex
 *                     (includes hard_certified)
 *   exact_pass        answered by the exact pass
 * soft_certified + exact_pass = Q.
 */
typedef struct {
    int32_t unanswered, ladder_overflows, hard_certified, soft_certified, exact_pass;
} ralm_counters_t;
ralm_status ralm_workspace_counters(const void *workspace, void *stream, ralm_counters_t *out);

/*
 * How full the candidate lists got in the LAST ralm_retrieve_topk_ex / _seq
 * call on this workspace: entries[i] = over all queries, the entries their
 * lists held when stage i of the ladder ended (the at most k' kept from the
 * stages before plus the scores the stage admitted), i < *n_stages; the other
 * elements are set to 0.  entries is a HOST array of RALM_MAX_LADDER_STAGES
 * elements; of a longer ladder (the sequential form) the first
 * RALM_MAX_LADDER_STAGES stages are reported.  Synchronises `stream`.  A
 * diagnostic: with rows in an order that the strided samples represent well a
 * stage that multiplies the rows scanned by g admits about r (g - 1) scores
 * per query, r <= k' the rank of its admission score (ralm_retrieve_topk_ex).
 */
#define RALM_MAX_LADDER_STAGES 40
ralm_status ralm_workspace_stage_entries(const void *workspace, void *stream, int32_t *n_stages,
                                         int64_t *entries);

/*
 * Which scan kernel each stage of a ralm_retrieve_topk_ex call with these
 * arguments takes, under the present reserve of compute units: routes[i],
 * i < *n_stages, is RALM_SCAN_*, and 0 for a stage that has no rows to scan and
 * for all elements behind.  routes is a HOST array of RALM_MAX_LADDER_STAGES
 * elements.  Nothing is launched or read (of the datastore's pointers only the
 * alignment counts), and no GPU is needed: without one the answer is that of a
 * device with 256 compute units.  A diagnostic.
 */
enum {
    RALM_SCAN_ALL = 1,           /* keeps every score (the first stage) */
    RALM_SCAN_ALL_QUARTERS = 2,  /* the same in tiles of 64 rows */
    RALM_SCAN_COUNTED = 3,       /* thresholds that admit many scores of a tile: counted per query, then stored */
    RALM_SCAN_PARKED = 4,        /* thresholds that admit few: collected one by one */
    RALM_SCAN_HELD = 5           /* the same, with the queries held in registers */
};
ralm_status ralm_scan_routes(int64_t Q, const ralm_datastore_t *ds, int32_t k, int32_t k_prime,
                             int32_t *n_stages, int32_t *routes);

/*
 * Whether the first stage of such a call (RALM_SCAN_ALL or
 * RALM_SCAN_ALL_QUARTERS) leaves bare scores and the best of every 32 rows, of
 * which its select reads few (*scores_only = 1), or a key per row (0).  Host
 * only, as ralm_scan_routes.  A diagnostic.
 */
ralm_status ralm_first_stage_scores(int64_t Q, const ralm_datastore_t *ds, int32_t k, int32_t k_prime,
                                    int32_t *scores_only);

/*
 * Build the low-precision scan copy of a datastore: dst[j, c] = round-to-
 * nearest-even(src[j, c]) in dst_dtype (RALM_BF16 or RALM_F16).  src is device
 * fp32 [N, d] with pitch src_stride elements, dst device [N, d] with pitch
 * dst_stride elements (0 = d for both).
 */
ralm_status ralm_build_scan_copy(const float *src, int64_t src_stride, void *dst, int32_t dst_dtype,
                                 int64_t dst_stride, int64_t N, int32_t d, void *stream);

/*
 * Scan copy for RALM_METRIC_L2: dst[j, 0..d) = round-to-nearest-even(src[j, c])
 * in dst_dtype; dst[j, d] + dst[j, d+1] = |src_j|^2 (summed in double, split
 * into a rounded head and the rounded remainder); dst[j, d+2 .. d+8) = 0.
 * src is device fp32 or fp16 [N, d] (src_dtype), dst device [N, d + 8] bf16 or
 * fp16; strides in elements (0 = d, d + 8).  src == dst is allowed for fp16
 * keys stored with a pitch of at least d + 8 that serve as their own scan
 * copy: then only the 8 extra columns are written.
 */
ralm_status ralm_build_scan_copy_l2(const void *src, int32_t src_dtype, int64_t src_stride, void *dst,
                                    int32_t dst_dtype, int64_t dst_stride, int64_t N, int32_t d,
                                    void *stream);

/*
 * Speculative retrieval from the per-request local caches (Alg. 1, the
 * speculative retrieval step; Section 3 "Speculative retrieval"; Fig. 2: the
 * cache is ranked with the retriever's own metric).  A cache holds datastore
 * row ids; the key is re-read from the exact datastore so that a cached
 * entry's score is the double sum, rounded once, that the knowledge-base
 * retrieval forms (the additions may come in another order).  This is what
 * makes the cache top-1 equal the knowledge-base top-1 whenever the latter is
 * cached.
 *
 *   cache_ids  device int32 [R, C]; request r owns entries [0, cache_len[r])
 *              of row r; every owned id must be in [0, N) (ids outside are
 *              skipped)
 *   cache_len  device int32 [R]; values are clamped to [0, C]
 *   queries    device fp32 [Qt, d]; request r owns rows q_offsets[r] ..
 *              q_offsets[r+1] (its speculation steps, in order)
 *   q_offsets  device int64 [R+1], non-decreasing, within [0, Qt].  Device
 *              data cannot be checked on the host: the kernel clamps each
 *              range to [0, Qt] and treats a decreasing pair as empty.
 *   spec_ids   device int32 [Qt]: top-1 cached id per query (-1 if the cache
 *              is empty);  spec_scores device fp32 [Qt] (-inf if empty).
 *              Rows of [0, Qt) that no request owns are left untouched.
 *   workspace  optional device scratch (may be NULL) of at least
 *              ralm_cache_lookup_workspace_bytes(Qt) = 8 bytes per query,
 *              8-byte aligned, contents undefined between calls.  Without it
 *              one workgroup serves a request, which leaves most of the chip
 *              idle when there are few requests (a single request with 4096
 *              cached rows then takes ~0.4 ms); with it the caches of up to
 *              512 requests are each split over several workgroups, where that
 *              fills the chip better, that merge through the workspace and the
 *              outputs (same results; ralm_lookup_route tells how many).
 */
size_t ralm_cache_lookup_workspace_bytes(int64_t Qt);
ralm_status ralm_cache_lookup(const int32_t *cache_ids, const int32_t *cache_len, int32_t C, int64_t R,
                              const float *queries, int64_t Qt, const int64_t *q_offsets,
                              const ralm_datastore_t *ds, int32_t *spec_ids, float *spec_scores,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * ralm_cache_lookup that writes every row of the outputs: rows of [0, Qt) that no
 * request owns get id -1 / score -inf, by the lookup itself or in a launch that it
 * needs anyway, so outputs need not be filled beforehand.
 */
ralm_status ralm_cache_lookup_all(const int32_t *cache_ids, const int32_t *cache_len, int32_t C, int64_t R,
                                  const float *queries, int64_t Qt, const int64_t *q_offsets,
                                  const ralm_datastore_t *ds, int32_t *spec_ids, float *spec_scores,
                                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * ralm_cache_lookup for callers that can neither allocate device memory nor
 * pass a workspace: code recorded under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation.  Same arguments and same results as
 * ralm_cache_lookup called with a workspace; the merge slots (8 bytes per
 * query) live in an array inside the library instead, 512 KiB per GPU, held
 * until the process ends.  Limit: Qt <= 65536 (RALM_ERR_RANGE beyond it).  The
 * call allocates nothing and only launches kernels (the slots are cleared by a
 * kernel).  All calls on one GPU share that array: two calls that overlap in
 * time on the same GPU (different streams or threads) race; calls ordered on
 * one stream are fine.
 */
#define RALM_STATIC_LOOKUP_MAX_QT 65536
ralm_status ralm_cache_lookup_static(const int32_t *cache_ids, const int32_t *cache_len, int32_t C, int64_t R,
                                     const float *queries, int64_t Qt, const int64_t *q_offsets,
                                     const ralm_datastore_t *ds, int32_t *spec_ids, float *spec_scores,
                                     void *stream);

/*
 * Speculative retrieval of k entries from the local caches (Section 5.3: KNN-LM
 * forms its next-token distribution from k retrieved entries, so its
 * speculation step needs the k best CACHED entries; ranked with the
 * retriever's own metric like every cache retrieval, Section 3 / Fig. 2).
 * Arguments as ralm_cache_lookup, plus
 *
 *   k           1 <= k <= min(C, RALM_MAX_K); C <= RALM_MAX_K_PRIME
 *   out_ids / out_scores  device [Qt, k], best first; ranks beyond the number
 *               of (valid) cached ids get id -1 / score -inf, as do queries
 *               that no request owns
 *   workspace   device scratch, 256-byte aligned, at least
 *               ralm_cache_lookup_topk_workspace_bytes(Qt, C)
 *
 * Cached ids must be distinct within a request (a repeated id is returned
 * repeatedly).  Feeds ralm_knnlm_probs directly.
 */
size_t ralm_cache_lookup_topk_workspace_bytes(int64_t Qt, int32_t C);
ralm_status ralm_cache_lookup_topk(const int32_t *cache_ids, const int32_t *cache_len, int32_t C, int64_t R,
                                   const float *queries, int64_t Qt, const int64_t *q_offsets,
                                   const ralm_datastore_t *ds, int32_t k, int32_t *out_ids,
                                   float *out_scores, void *workspace, size_t workspace_bytes, void *stream);

/*
 * How a cache lookup with these arguments is launched.  k = 0: ralm_cache_lookup_all
 * with a workspace; k > 0: ralm_cache_lookup_topk.  workgroups: per request
 * (0: the rows go through the re-score of a retrieval instead).  pieces: 16-byte
 * pieces of a row that a lane of the matrix-core form has in flight (0: the vector
 * units read the rows).  clears: 1 if a launch of its own clears merge slots or
 * answers the queries that no request owns (0 for k > 0).  All three are HOST
 * pointers; nothing is launched or read (of the datastore's pointers only the
 * alignment counts), and no GPU is needed.  A diagnostic.
 */
ralm_status ralm_lookup_route(int64_t R, int64_t Qt, int32_t C, const ralm_datastore_t *ds, int32_t k,
                              int32_t *workgroups, int32_t *pieces, int32_t *clears);

/*
 * Verification compare (Alg. 1: m = argmin_i d^_i != d_i).  For request r with
 * stride s_r = q_offsets[r+1] - q_offsets[r]:
 *   first_mismatch[r] = min { i in [0, s_r) : spec_ids[q_offsets[r] + i] !=
 *                             true_ids[(q_offsets[r] + i) * true_stride] }
 * or s_r when every step matches (0-based; s_r = 0 gives 0).  true_stride = k
 * reads the rank-0 column of a [Q, k] retrieval result in place.
 *
 *   spec_ids   device int32 [Qt];  true_ids device int32 [Qt * true_stride];
 *   q_offsets  device int64 [R+1] (clamped as in ralm_cache_lookup);
 *   first_mismatch  device int32 [R]
 */
ralm_status ralm_verify(const int32_t *spec_ids, const int32_t *true_ids, int64_t true_stride,
                        int64_t Qt, const int64_t *q_offsets, int64_t R, int32_t *first_mismatch,
                        void *stream);

/*
 * Cache update after a verification step (Alg. 1, Q.insert(C.retrieve(..));
 * Section 3 "Batched verification": top-1 update and top-k update =
 * prefetching, Fig. 2; Section 5.3: for KNN-LM the next n entries after a
 * retrieved one).  The paper's cache has no stated capacity; here a request's
 * cache is a ring of C ids: an id that is already cached is not inserted
 * again, and once all C slots are used the oldest inserted id is overwritten.
 *
 *   cache_ids / cache_len   device int32 [R, C] / [R], as in ralm_cache_lookup;
 *                           updated in place.  Owned ids must be distinct.
 *   cache_head  device int32 [R]: the slot that the next insertion into a FULL
 *               cache overwrites; start with zeros; updated in place.
 *   true_ids    device int32: rank-j id of query q at true_ids[q * true_stride
 *               + j] (the out_ids of a retrieval with k = true_stride)
 *   q_offsets   device int64 [R+1] (clamped as in ralm_cache_lookup)
 *   first_mismatch  device int32 [R] from ralm_verify, or NULL.  Given: only
 *               the steps 0 .. min(first_mismatch[r], s_r - 1) of request r are
 *               taken (the later ones were retrieved for a context that is
 *               rolled back).  NULL: all s_r steps.
 *   p           ranks 0 .. p-1 of each taken step are taken (1 = top-1 update,
 *               20 = the paper's prefetch size); 1 <= p <= true_stride
 *   n_next      0: a taken id t is itself the candidate; n > 0: its successors
 *               t+1 .. t+n are (spatial locality of KNN-LM datastores)
 *   N           candidates outside [0, N) are dropped, as are negative ids
 *
 * Candidates are inserted in the order step, rank, successor; the result is
 * that of doing so one at a time.  Requests are independent (one workgroup
 * each, 64 candidates at a time).  Cost per candidate grows with the number of
 * cached ids (linear membership test over the row in LDS); ranks without an id
 * and successors outside [0, N) cost next to nothing; C <= 16384.
 */
ralm_status ralm_cache_insert(int32_t *cache_ids, int32_t *cache_len, int32_t *cache_head, int32_t C,
                              int64_t R, const int32_t *true_ids, int64_t true_stride, int64_t Qt,
                              const int64_t *q_offsets, const int32_t *first_mismatch, int32_t p,
                              int32_t n_next, int64_t N, void *stream);

/*
 * KNN-LM neighbour distribution (Section 5.3: a distribution over the target
 * tokens of the k retrieved entries, computed from their distances).  Input is
 * the output of a retrieval: ids / scores device [Q, k], a larger score being a
 * closer entry.
 *
 *   values       device int32 [N]: target token of every datastore entry
 *   temperature  T > 0; weight_i = exp(score_i / T) / sum_j exp(score_j / T)
 *   out_tokens   device int32 [Q, k]: values[ids]  (-1 for an unfilled entry:
 *                id < 0 or >= N; its weight is 0)
 *   out_weights  device fp32 [Q, k], each row sums to 1
 *   out_top_token / out_top_prob  optional device [Q] (either may be NULL): the
 *                token with the largest summed weight and that sum; the smaller
 *                token id on ties; -1 / 0 for a query without filled entries.
 * Sums and exponentials are formed in double and rounded once to fp32.
 */
ralm_status ralm_knnlm_probs(const int32_t *ids, const float *scores, int64_t Q, int32_t k,
                             const int32_t *values, int64_t N, float temperature, int32_t *out_tokens,
                             float *out_weights, int32_t *out_top_token, float *out_top_prob,
                             void *stream);

/*
 * The generator's cache of keys and values, in 4 bits and in pages.
 *
 * A request's tokens lie in pages of page_tokens tokens; a page holds them for
 * all layers and heads, so that forking, rolling back and copying a context is
 * one operation for all layers.  Which pages are whose:
 *
 *   table  device int32 [R, max_pages]: the page of the request's tokens
 *          page_tokens * j .. ; -1 behind its last page
 *   lens   device int32 [R]: tokens of the request
 *   refs   device int32 [n_pages]: how many places of the table hold the page;
 *          0 = free (append, read, attention and copy_pages do not use it: NULL)
 *   pages  device, n_pages * ralm_kv_page_bytes() bytes, 16-byte aligned
 *
 * A new cache is lens = refs = 0 and table = -1; its pages need no clearing.
 * d is 64, 128 or 256; page_tokens a power of two in [16, 256]; n_pages <=
 * 2^22, R <= 2^16, max_pages * page_tokens <= 2^30.
 *
 * Format: 32 neighbouring numbers of a head share a power of two 2^e, stored as
 * e + 127 in a byte, and each is one of +-{0, .5, 1, 1.5, 2, 3, 4, 6} * 2^e: 4.25
 * bits a number.  e is the smallest integer in [-126, 125] with max|x| <= 6 * 2^e
 * (125 beyond 6 * 2^125, so that what is finite stays so in fp32 and bf16), a number
 * becomes the nearest of the sixteen, ties to the even code (0, 1, 2, 4).
 * A block that holds an infinity or NaN gets the byte 255 and stands for NaN.
 * fp32, bf16 and fp16 inputs of equal value give equal codes.  (Layout of a page:
 * [layer][head][page_tokens / 16][17 d] bytes; kv_kernels.h has the rest.)
 *
 * Table entries outside [0, n_pages) are no places: tokens there are not stored,
 * read as zeros and not attended to.  Pages of one request must be distinct, and
 * a page that another request shares must not be appended to: ralm_kv_reserve
 * sees to both.
 */
typedef struct {
    void *pages;
    int64_t n_pages;
    int32_t n_layers, n_heads, d, page_tokens;
    int32_t *table;
    int32_t *lens;
    int32_t *refs;
    int64_t R;
    int32_t max_pages;
} ralm_kv_t;

/* Bytes of a page; 0 for arguments out of range. */
size_t ralm_kv_page_bytes(int32_t n_layers, int32_t n_heads, int32_t d, int32_t page_tokens);

/*
 * Keys and values of new tokens into the cache of a layer, and out of it.
 *
 *   k, v       device [n, n_heads, d] of dtype (fp32, bf16 or fp16); strides in
 *              elements from token to token and head to head (0: dense);
 *              bases and strides multiples of 16 bytes
 *   offsets    device int64 [R+1], non-decreasing: rows offsets[r] ..
 *              offsets[r+1]-1 are request r's
 *   append     they are the request's last tokens: row i of s goes to place
 *              lens[r] - s + i (ralm_kv_reserve has made the room and moved lens)
 *   read       from place start[r] on (device int32 [R]), or the last ones too
 *              (start == NULL).  fp16 overflows to infinity beyond its range.
 *
 * Rows of no request are neither stored nor written; places outside the table
 * are not stored and read as zeros.
 */
ralm_status ralm_kv_append(const ralm_kv_t *kv, int32_t layer, const void *k, const void *v, int32_t dtype,
                           int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                           int64_t v_head_stride, const int64_t *offsets, int64_t n, void *stream);
ralm_status ralm_kv_read(const ralm_kv_t *kv, int32_t layer, const int64_t *offsets, int64_t n,
                         const int32_t *start, void *k, void *v, int32_t dtype, int64_t k_token_stride,
                         int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                         void *stream);

/*
 * Attention of every request's last tokens over its cache:
 *
 *   out[i, h] = sum_j softmax_j(scale * q[i, h] . K[j, h / G]) V[j, h / G],   G = n_q_heads / n_heads
 *
 * over the tokens j that query i sees.  The s_r = offsets[r+1] - offsets[r]
 * queries of request r stand at its last places p = lens[r] - s_r + i, their own
 * keys and values having been appended; they see j <= p, and with window > 0 of
 * those only j > p - window and the first `sinks` tokens.  One token per request,
 * drafted tokens and chunks of a prompt are the same call.
 *
 *   q, out     device [Qt, n_q_heads, d], bf16 or fp16; strides in elements
 *              (0: dense), multiples of 8; bases 16-byte aligned
 *   max_q, max_len  the largest s_r and lens[r], as far as the host knows them:
 *              they choose the launch.  0 is unknown, and so is a max_q beyond Qt:
 *              the launch is then one for the mean Qt / R, and for the table's width.
 *              Smaller or larger than the truth, or unknown, they cost time, never a
 *              result.
 *   lse        device fp32 [Qt, n_q_heads] or NULL: log sum exp of a row's scores
 *   workspace  ralm_kv_attention_workspace_bytes(), 16-byte aligned (may be NULL
 *              where that is 256): sums of contexts that are split over workgroups
 *
 * A row that sees nothing (lens[r] < s_r) is 0, its lse -inf.  Scores and sums
 * are fp32; weights are rounded to 8 bits (bf16) or 16 bits (fp16) for their
 * product with V.  A key that is NaN makes the rows that see it NaN, a value the
 * 32 numbers of its block; rows that do not see it are not touched.  Results are
 * the same from call to call.  R * n_heads <= 2^23 - 8, Qt * n_q_heads <= 2^30.
 */
size_t ralm_kv_attention_workspace_bytes(const ralm_kv_t *kv, int32_t n_q_heads, int64_t Qt, int64_t max_q,
                                         int64_t max_len, int32_t window, int32_t sinks);
ralm_status ralm_kv_attention(const ralm_kv_t *kv, int32_t layer, const void *q, int32_t dtype,
                              int64_t q_token_stride, int64_t q_head_stride, int32_t n_q_heads,
                              const int64_t *offsets, int64_t Qt, int64_t max_q, int64_t max_len, float scale,
                              int32_t window, int32_t sinks, void *out, int64_t out_token_stride,
                              int64_t out_head_stride, float *lse, void *workspace, size_t workspace_bytes,
                              void *stream);

/*
 * Pages.  The free page that is taken is always the one with the lowest id, so
 * the state behind a call follows from the state before it.  All of them work on
 * kv's table, lens and refs in place, on the device, without the host knowing
 * any length.  Workspace: ralm_kv_pages_workspace_bytes(), 16-byte aligned.
 *
 * ralm_kv_reserve  room for grow[r] more tokens (device int32 [R]; <= 0: none) of
 *   every request, lens[r] += grow[r].  New pages are taken in the order of the
 *   requests; a last page that is partly filled and shared (its count above 1
 *   when the call begins) is copied to a page of the request's own first.  A
 *   request is served if the pages needed up to and with it are there (or it
 *   needs none); others, and those that would outgrow the table, stay as they are.
 *   granted: device int32 [R] or NULL, 1 or 0.
 * ralm_kv_fork  for i < n: request dst[i], which must be empty, shares the pages
 *   of src[i]'s first keep[i] tokens (keep NULL: all).  Pairs whose dst is not
 *   empty or whose ids are out of range or equal are left out; a dst comes once in
 *   a call and is no src of it.
 * ralm_kv_truncate  lens[r] = min(lens[r], new_lens[r]); pages behind it are let
 *   go, and free when nobody else holds them.  0 ends a request; the
 *   first_mismatch of a verification rolls it back.
 * ralm_kv_copy_pages  contents of page src[i] to page dst[i], i < n; no dst may be
 *   a src or come twice.  Ids out of range are left out.
 * ralm_kv_compact  the n pages in use become pages 0 .. n-1: those at n and behind,
 *   in order, take the free places in front, in order.  The new table, counts and n
 *   go to table_out [R, max_pages], refs_out [n_pages], used [1]; they may be the
 *   cache's own.  If they are not, the old table stays valid (nothing of what it
 *   names is overwritten) until the new counts are used to reserve.
 */
size_t ralm_kv_pages_workspace_bytes(const ralm_kv_t *kv);
ralm_status ralm_kv_reserve(const ralm_kv_t *kv, const int32_t *grow, int32_t *granted, void *workspace,
                            size_t workspace_bytes, void *stream);
ralm_status ralm_kv_fork(const ralm_kv_t *kv, const int32_t *src, const int32_t *dst, const int32_t *keep,
                         int64_t n, void *stream);
ralm_status ralm_kv_truncate(const ralm_kv_t *kv, const int32_t *new_lens, void *stream);
ralm_status ralm_kv_copy_pages(const ralm_kv_t *kv, const int32_t *src, const int32_t *dst, int64_t n, void *stream);
ralm_status ralm_kv_compact(const ralm_kv_t *kv, int32_t *table_out, int32_t *refs_out, int32_t *used,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * Verification of drafted tokens by a target's probabilities (the sampled form
 * of ralm_verify's compare: the tokens that come out are distributed as the
 * target's own).  Request r drafted s_r = q_offsets[r+1] - q_offsets[r] tokens.
 *
 *   draft_ids     device int32 [Qt]
 *   draft_probs   device [Qt, V], what they were drawn from; NULL: every draft is
 *                 certain (a greedy draft, a neighbour's token)
 *   target_probs  device [Qt + R, V]: row q_offsets[r] + r + i belongs to the i-th
 *                 draft of request r, row i = s_r to the token behind them
 *   *_stride      elements from row to row (0 = V); dtype fp32, bf16 or fp16 for both
 *   u [Qt], u_next [R]  device fp32, uniform in [0, 1)
 *   accepted      device int32 [R]: the first i with u_i q_i(x_i) >= p_i(x_i), or s_r
 *   next_token    device int32 [R]: drawn by u_next from max(p - q, 0) of that row (from
 *                 p if nothing is left, or behind s_r accepted ones); -1 if p is 0 too
 *   workspace     ralm_verify_draft_workspace_bytes(), 16-byte aligned
 *
 * Defined in whole numbers, so that it does not depend on how sums are formed: P =
 * floor(min(max(p, 0), 1) * 2^36), Q alike, m = floor(u * 2^24); accepted while
 * m Q < 2^24 P; w = max(P - Q, 0), S = sum w; the next token is the smallest v with
 * w_0 + .. + w_v > floor(m S / 2^24).  NaN counts as 0, a draft outside [0, V) is not accepted.
 * R <= 2^16, V <= RALM_MAX_VOCABULARY.
 */
#define RALM_MAX_VOCABULARY (1 << 20)
size_t ralm_verify_draft_workspace_bytes(int64_t R, int32_t V);
ralm_status ralm_verify_draft(const int32_t *draft_ids, const void *draft_probs, int64_t draft_stride,
                              const void *target_probs, int64_t target_stride, int32_t dtype, int32_t V,
                              const float *u, const float *u_next, int64_t Qt, const int64_t *q_offsets,
                              int64_t R, int32_t *accepted, int32_t *next_token, void *workspace,
                              size_t workspace_bytes, void *stream);

/*
 * The rest of the generator's decoder: the products, norms and positions around
 * its attention, and the distribution that its drafts are verified against.
 *
 * ralm_linear  rows times weights, and what usually follows at once:
 *
 *     out[i, n] = residual[i, n] + act(x[i] . w[n] + bias[n])                                            gated = 0
 *     out[i, n] = residual[i, n] + act(x[i] . w[n] + bias[n]) * (x[i] . w[N + n] + bias[N + n])          gated = 1
 *
 *   x          device [T, K] of dtype (bf16 or fp16), rows x_stride elements apart
 *   w          device [N, K] of dtype ([2N, K] if gated), rows w_stride apart
 *   bias       device [N] ([2N]) of dtype, or NULL
 *   act        RALM_ACT_*; gelu is x Phi(x), gelu_tanh its usual approximation,
 *              silu x / (1 + exp(-x)).  gelu is good to 2^-20 of its value where out is fp32, to
 *              2^-17 before the rounding to 16 bits; silu and gelu_tanh, which are x / (1 + exp(e)),
 *              to 2^-21 (1 + |e|) of theirs; all down to 2^-118
 *   residual   device [T, N] of out_dtype, or NULL; it may be out itself (same
 *              stride), and must not overlap it otherwise
 *   out        device [T, N] of out_dtype (dtype or fp32); must not overlap x, w or bias
 *   workspace  16-byte aligned, sums of products that are split over workgroups:
 *              ralm_linear_workspace_bytes() of T or more rows, a search on the host (0.1 ms for 256 rows, 0.3 ms for 8192)
 *              for what is enough for all calls of up to so many; or
 *              ralm_linear_workspace_bytes_exact(), what a call of exactly T rows needs (fewer rows may need more).
 *              May be NULL where that is 0
 *
 * Strides of 0 are dense.  K is a multiple of 8 in [8, 2^17]; x and w are 16-byte
 * aligned and their strides multiples of 8 elements, at most 2^22; out, residual
 * and bias are aligned to their type.  T <= 2^22, N <= 2^20 (2^19 gated), T x N <= 2^36 (2^35).
 * Products are exact and summed in fp32, everything up to the one rounding to
 * out_dtype is fp32.  Results are the same from call to call; they may differ in
 * the last bits with T, which chooses how a sum is split.
 */
enum { RALM_ACT_NONE = 0, RALM_ACT_RELU = 1, RALM_ACT_GELU = 2, RALM_ACT_GELU_TANH = 3, RALM_ACT_SILU = 4 };
size_t ralm_linear_workspace_bytes(int64_t T, int32_t N, int32_t K, int32_t gated);
size_t ralm_linear_workspace_bytes_exact(int64_t T, int32_t N, int32_t K, int32_t gated);
ralm_status ralm_linear(const void *x, int64_t x_stride, int64_t T, const void *w, int64_t w_stride, int32_t N,
                        int32_t K, int32_t dtype, const void *bias, int32_t act, int32_t gated,
                        const void *residual, int64_t residual_stride, void *out, int64_t out_stride,
                        int32_t out_dtype, void *workspace, size_t workspace_bytes, void *stream);

/*
 * A block's output into the residual stream, and the stream's norm for the next block:
 *
 *     y = x, or norm(x) * post_weight + post_bias with post = 1
 *     s = residual + scale * gate * y
 *     out = norm(s) * weight + bias
 *
 *   kind RALM_NORM_RMS:    norm(y) = y / sqrt(mean(y^2) + eps)
 *   kind RALM_NORM_LAYER:  norm(y) = (y - mean(y)) / sqrt(mean((y - mean(y))^2) + eps)
 *
 *   x          device [T, D] of x_dtype
 *   post_weight, post_bias, weight, bias   device [D] of param_dtype; NULL: 1 and 0
 *   gate       device of x_dtype or NULL (1): [D] with gate_rows = 0, [T, D] with 1
 *   residual   device [T, D] of sum_dtype or NULL (0)
 *   sum        device [T, D] of sum_dtype, or NULL (s is not wanted); may be residual
 *              or x itself (same type and stride)
 *   out        device [T, D] of out_dtype, or NULL (only s is wanted); may be x
 *
 * Apart from that outputs overlap no input and not each other.  Types are fp32, bf16 or fp16, pointers
 * aligned to them; strides in elements, 0 = dense.  1 <= D <= RALM_MAX_NORM, T <= 2^22, T x D <= 2^36.  Statistics and everything
 * in between are fp32; the norm is taken of s before it is rounded.
 */
enum { RALM_NORM_RMS = 0, RALM_NORM_LAYER = 1 };
#define RALM_MAX_NORM 32768
typedef struct {
    int64_t T;
    int32_t D, kind;
    float eps, scale;
    const void *x;
    int64_t x_stride;
    int32_t x_dtype, param_dtype;
    int32_t post;
    const void *post_weight, *post_bias;
    const void *gate;
    int64_t gate_stride;
    int32_t gate_rows;
    const void *residual;
    int64_t residual_stride;
    void *sum;
    int64_t sum_stride;
    int32_t sum_dtype;
    const void *weight, *bias;
    void *out;
    int64_t out_stride;
    int32_t out_dtype;
} ralm_norm_t;
ralm_status ralm_residual_norm(const ralm_norm_t *norm, void *stream);

/*
 * Rotary positions.  Two numbers a, b of a head that turn together become
 *
 *     (a cos t - b sin t) * amplitude,  (b cos t + a sin t) * amplitude,       t = place * freqs[j]
 *
 * for the pairs j < rot / 2: the numbers j and j + rot / 2 of the head (interleaved = 0) or
 * 2 j and 2 j + 1 (interleaved = 1); the numbers from rot on stay.
 *
 * ralm_kv_append_rotary  ralm_kv_append with the keys turned on the way in, and
 *   the queries of the same tokens turned:
 *   q, q_out   device [n, n_q_heads, d] of dtype; q_out may be q itself (same
 *              strides) and must overlap no input otherwise.  q NULL: keys and values alone
 *   k, v, offsets, n, strides   as in ralm_kv_append
 *   freqs      device fp64 [rot / 2], radians per place; rot even, 0 <= rot <= d
 *   shift      device int32 [R] or NULL: a token's place is its place in the cache
 *              (lens[r] - s + i) plus shift[r]
 *   Angles, turns and their sums are formed in fp64 and rounded to dtype by way of
 *   fp32, so that a key's codes do not depend on how its turn is formed: the
 *   cache holds what ralm_kv_append stores of the turned keys.  Queries of no request are not written.
 *
 * ralm_rotary_frequencies  (host, no GPU) fp64 frequencies of a plain or scaled base:
 *   freqs[j] = f_j (m + (1 - m) / factor),  f_j = base^(-2 j / rot),
 *   m = clamp((context f_j / 2 pi - low) / (high - low), 0, 1): pairs that turn at
 *   least `high` times within the `context` tokens of the training stay as they are, those that turn
 *   at most `low` times are slowed down by factor.  context = 0: m = 0 for all.
 */
ralm_status ralm_kv_append_rotary(const ralm_kv_t *kv, int32_t layer, const void *q, int64_t q_token_stride,
                                  int64_t q_head_stride, int32_t n_q_heads, void *q_out, int64_t q_out_token_stride,
                                  int64_t q_out_head_stride, const void *k, const void *v, int32_t dtype,
                                  int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                  int64_t v_head_stride, const double *freqs, int32_t rot, int32_t interleaved,
                                  double amplitude, const int32_t *shift, const int64_t *offsets, int64_t n,
                                  void *stream);
ralm_status ralm_rotary_frequencies(double *freqs, int32_t rot, double base, double factor, double context,
                                    double low, double high);

/*
 * The target of a verification: the model's distribution mixed with the neighbours'
 * (Section 5.3; the interpolation of KNN-LM),
 *
 *   out[i, v] = (1 - share_i) softmax(logits[i] / temperature)[v] + share_i sum_{j: tokens[i, j] = v} weights[i, j]
 *
 *   logits     device [Q, V] of dtype (fp32, bf16, fp16), rows logits_stride elements apart (0: V)
 *   tokens, weights   device int32, fp32 [Q, k] (of ralm_knnlm_probs); tokens outside
 *              [0, V) count for nothing.  0 <= k <= RALM_MAX_K
 *   share      device fp32 [Q] or NULL: share_all for every row
 *   out        device [Q, V] of out_dtype; may be logits itself (same type and stride)
 *   workspace  ralm_knnlm_target_workspace_bytes() of Q or more rows, 16-byte aligned (may be NULL where that is 0)
 *
 * Sums and exponentials are fp32, a token's weights are added in the order of j, one
 * rounding to out_dtype.  Logits of -inf are probabilities of 0; a row of nothing
 * else has the neighbours' part alone.  +inf or NaN make their row NaN.  V <= RALM_MAX_VOCABULARY,
 * Q <= 2^20; where V is more than 65536, Q x V, V rounded up to
 * a multiple of 4096, is below 2^36.  Probabilities below 2^-126 may be 0.
 */
size_t ralm_knnlm_target_workspace_bytes(int64_t Q, int32_t V);
ralm_status ralm_knnlm_target(const void *logits, int64_t logits_stride, int64_t Q, int32_t V, int32_t dtype,
                              float temperature, const int32_t *tokens, const float *weights, int32_t k,
                              const float *share, float share_all, void *out, int64_t out_stride,
                              int32_t out_dtype, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Optimal speculation stride scheduler, OS^3 (Section 4; estimation of its
 * parameters: Appendix A.2, "Parameter estimation").  Host-only scalar
 * functions; every pointer is a HOST pointer; nothing is launched.
 *
 * ralm_os3_gamma: estimate of the speculation accuracy gamma from the w most
 *   recent verification steps of a request: strides[t] = s(t), matched[t] =
 *   M(s(t)) = number of speculated documents that matched before the first
 *   mismatch (the first_mismatch of ralm_verify):
 *       gamma^ = sum_t M(t) / ( sum_t M(t) + #{t : M(t) < s(t)} ),
 *   truncated at gamma_max (the paper uses w = 5, gamma_max = 0.6).  0 when
 *   there is no history (w <= 0) or nothing matched.
 * ralm_os3_objective: expected verified documents per unit time for stride s,
 *       (1 - gamma^s) / (1 - gamma) / latency(s),
 *   latency(s) = s a + b (synchronous verification; async == 0), or
 *   gamma^s ((s-1) a + max(a, b)) + (1 - gamma^s)(s a + b) (asynchronous),
 *   with a = latency of a speculation step, b = latency of a verification
 *   step.  The expectation is formed as the sum of gamma^i, i < s, so gamma = 1
 *   needs no special case.  NaN for s < 1, negative a or b, gamma outside [0, 1].
 * ralm_os3_stride: the s in [1, s_max] with the largest objective; the
 *   smallest such s on ties.
 * ralm_os3_latency: a (or b) as the mean of the n most recent measurements
 *   (Appendix A.2 estimates both from recent profiling and fixes no window
 *   length); 0 for n <= 0.
 * ralm_os3_next_stride: the stride for the next round from a request's history:
 *   gamma^ from (strides, matched, w), a and b from their samples, then
 *   ralm_os3_stride.  1 while any of the three histories is empty (the paper
 *   starts with s = 1).
 */
double ralm_os3_gamma(const int32_t *strides, const int32_t *matched, int32_t w, double gamma_max);
double ralm_os3_objective(double gamma, double a, double b, int32_t s, int32_t async);
int32_t ralm_os3_stride(double gamma, double a, double b, int32_t s_max, int32_t async);
double ralm_os3_latency(const double *samples, int32_t n);
int32_t ralm_os3_next_stride(const int32_t *strides, const int32_t *matched, int32_t w,
                             const double *a_samples, int32_t n_a, const double *b_samples, int32_t n_b,
                             double gamma_max, int32_t s_max, int32_t async);

/*
 * Asynchronous verification (Section 3, "Asynchronous verification"; latency
 * model of Section 4: a verification that overlaps the next speculation step
 * costs (s-1) a + max(a, b) instead of s a + b).  Every call here is ordered on
 * the caller's stream only, so the batched retrieval of step t and the cache
 * lookup of step t+1 can be issued on two streams.  The scan, however, runs as
 * a persistent grid whose workgroups fill the LDS of every compute unit (one
 * each, or two for batches of up to 32 queries over 16-bit rows), so
 * a kernel on another stream finds no free unit until a scan launch ends.
 * ralm_scan_reserve_cus(n) makes every later retrieval call of the process
 * launch its scans with at most 256 - n workgroups, rounded down to a multiple
 * of 8, so that n compute units stay free (n = 8: one per XCD; 0 restores the
 * default).  The scan slows down by about n / 256 (n = 8, 1024 queries over
 * 768 elements: 7 %, because four query tiles do not share out the units that
 * are left and the scan takes another kernel); batches of up to 32 queries put
 * one workgroup on a unit then, which leaves half of every unit's LDS free (4 %
 * slower); larger batches read the rows in more launches, none longer than half
 * of the scan, between which kernels that need more than n units get onto the
 * chip.  Process-wide setting, read when a call is issued.
 */
void ralm_scan_reserve_cus(int32_t n);

/*
 * Timing aid for benchmarks.  While enabled, ralm_retrieve_topk_ex brackets
 * each launch of its scan kernel (a call makes several: together they read
 * every row of the datastore exactly once) with HIP events on the call's
 * stream.  ralm_profile_scan_ms synchronises those events and returns the
 * total milliseconds and the number of bracketed launches since the last
 * reset (host pointers), then resets.  At most 2048 launches are recorded
 * between resets.  Not thread-safe; off by default.
 */
void ralm_profile_enable(int32_t on);
ralm_status ralm_profile_scan_ms(float *total_ms, int32_t *launches);

/* Text of the calling thread's last error (static storage; never NULL). */
const char *ralm_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* RALM_H */
