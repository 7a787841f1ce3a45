/*
 * plaid.h -- C ABI of the MI355X (gfx950) PLAID search library.
 *
 * The library runs the search pipeline of "PLAID: An Efficient Engine for Late Interaction
 * Retrieval" (Figure 4, Sections 4.1-4.5) for one or more queries on ONE GPU:
 *
 *   stage 1  S_cq = C . Q^T (Eq. 2); per query token the nprobe best centroids; candidate
 *            passages = union of the probed centroids' inverted lists (Section 4.1, no size cap);
 *   stage 2  centroid interaction (Eq. 3-4) over all candidates using only tokens whose centroid
 *            passes the pruning test max_i S_cq[c][i] >= t_cs (Eq. 5); keep the best ndocs;
 *   stage 3  centroid interaction without pruning over those; keep the best max(1, ndocs/4)
 *            (Figure 4, Section 4.3);
 *   stage 4  decompress the residuals of those passages through the byte lookup table
 *            (Section 4.5), exact MaxSim (Eq. 1), best k (Section 4.4).
 *
 * Readings where the paper is silent: rankings are by (score descending, id ascending); a passage
 * with no surviving token in stage 2 scores -infinity and still fills the ndocs slots in pid
 * order; reconstructed vectors are centroid + bucket weight with no renormalisation; packed
 * bucket indices are stored most-significant first (dimension order preserved inside a byte).
 *
 * Conventions: every function returns PLAID_OK (0) or a negative plaid_status and never throws
 * or aborts; plaid_last_error() returns a thread-local description of the last failure.
 * Pointers marked DEVICE are HIP device pointers valid on the index's device; pointers marked
 * HOST are ordinary host pointers.  The caller owns every buffer it passes; the library owns the
 * index handle and a per-index workspace that grows on demand and is released by
 * plaid_index_free.  Searches on one index must not run concurrently.  Kernels are enqueued on
 * the caller's stream; plaid_search returns without waiting for them unless stated otherwise.
 */
#ifndef PLAID_H
#define PLAID_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PLAID_QLEN 32 /* query tokens per query   */
#define PLAID_DIM 128 /* embedding dimension      */

typedef enum {
    PLAID_OK = 0,
    PLAID_EINVAL = -1,  /* null pointer, size out of range, malformed view */
    PLAID_ENOMEM = -2,  /* host or device allocation failed                */
    PLAID_EHIP = -3,    /* a HIP runtime call failed (text in last_error)  */
    PLAID_EIO = -4,     /* file could not be opened or read                */
    PLAID_EFORMAT = -5  /* file is not a PLAID index file                  */
} plaid_status;

typedef struct plaid_index plaid_index; /* opaque */

/* Borrowed description of an index (storage format of Section 3.1: a 4-byte centroid id and a
 * 16*nbits-byte packed residual per token; inverted lists of unique passage ids, Section 4.1).
 * All arrays live on the host (on_device = 0) or all on the device (on_device = 1). */
typedef struct {
    int32_t dim;                 /* must be PLAID_DIM */
    int32_t nbits;               /* 1 or 2 bits per residual dimension */
    int64_t num_centroids;       /* C, 1 <= C < 2^31 */
    int64_t num_passages;        /* P, 1 <= P < 2^31 */
    int64_t num_embeddings;      /* N = doc_offsets[P] */
    const float *centroids;      /* [C][128] row-major fp32 */
    const int64_t *doc_offsets;  /* [P+1], doc_offsets[0] = 0, non-decreasing; tokens of passage p are
                                    doc_offsets[p] .. doc_offsets[p+1]-1 */
    const int32_t *codes;        /* [N], centroid id of each token, in [0, C) */
    const uint8_t *residuals;    /* [N][16*nbits] packed bucket indices */
    const float *bucket_weights; /* [2^nbits] */
    const int64_t *ivf_offsets;  /* [C+1], ivf_offsets[0] = 0 */
    const int32_t *ivf_pids;     /* [ivf_offsets[C]], ascending unique pids per centroid */
    int32_t on_device;
} plaid_index_view;

/* Optional per-stage outputs of plaid_search_debug.  Every pointer is DEVICE, caller-owned, and may be
 * NULL (that output is skipped).  nq is the number of queries of the call. */
typedef struct {
    float *S_cq;          /* [nq][C][32]  Eq. 2 scores, row c = centroid c (the score kernel's values: see
                             plaid_get_score_kernel for how close to the definition's they are) */
    int32_t *probed;      /* [nq][32][nprobe]  per query token, best first (Section 4.1) */
    int32_t *cand;        /* [nq][P]  ascending candidate pids, first n_cand[q] valid */
    int32_t *n_cand;      /* [nq] */
    int32_t *sel2_ids;    /* [nq][ndocs]  stage-2 survivors, unspecified order, first n2[q] valid */
    float *sel2_scores;   /* [nq][ndocs]  their pruned centroid-interaction scores (Eq. 3-5) */
    int32_t *n2;          /* [nq]  = min(ndocs, n_cand) */
    int32_t *sel3_ids;    /* [nq][max(1,ndocs/4)]  stage-3 survivors, unspecified order */
    float *sel3_scores;   /* [nq][max(1,ndocs/4)]  their unpruned centroid-interaction scores (Eq. 3-4) */
    int32_t *n3;          /* [nq]  = min(max(1,ndocs/4), n2) */
    uint32_t *keep;       /* [nq][ceil(C/32)]  pruning map of Eq. 5: bit c%32 of word c/32 = centroid c is kept */
} plaid_debug_buffers;

/* Read an index file and upload it to `device` (a HIP device ordinal).  File layout, little-endian:
 * bytes 0-7 "PLAIDIX1"; int32 dim, int32 nbits, int64 C, P, N, ivf_len; zero padding to byte 64; then
 * centroids, doc_offsets, codes, residuals, bucket_weights, ivf_offsets, ivf_pids in the types of
 * plaid_index_view, each section starting at a multiple of 64 bytes.  On success *out is a new handle.
 * Errors: PLAID_EINVAL, PLAID_EIO, PLAID_EFORMAT, PLAID_ENOMEM, PLAID_EHIP. */
int plaid_index_load(const char *path, int device, plaid_index **out);

/* Build a handle from caller memory.  copy = 1: the arrays (host or device) are copied into
 * library-owned device memory.  copy = 0: requires on_device = 1; the library keeps the caller's device
 * pointers (centroids, codes and residuals must then be aligned to 16 bytes, else PLAID_EINVAL) and the caller
 * must keep them alive and unchanged until plaid_index_free.  The arrays are validated either way (offsets monotone
 * from 0 to their end, codes in [0, C), passage ids in [0, P) and strictly ascending within each list): on the host for
 * host arrays, by one kernel for device arrays; a violation is PLAID_EINVAL and nothing is searched. */
int plaid_index_from_view(const plaid_index_view *view, int device, int copy, plaid_index **out);

/* Release the handle, its workspace and any memory the library allocated for it.  NULL is allowed. */
void plaid_index_free(plaid_index *idx);

/* Search nq queries (Figure 4 pipeline, stages as listed at the top of this file).
 *   Q           DEVICE  [nq][32][128] fp32 query token embeddings (unit norm expected, not checked), 16-byte aligned
 *   nprobe      centroids probed per query token, 1 <= nprobe <= C
 *   t_cs        pruning threshold of Eq. 5; -INFINITY disables pruning, +INFINITY prunes everything
 *   ndocs       passages kept by stage 2 (>= 1); stage 3 keeps max(1, ndocs/4)
 *   k           results per query (>= 1)
 *   out_ids     DEVICE  [nq][k] passage ids, best first; unused slots -1
 *   out_scores  DEVICE  [nq][k] MaxSim scores (Eq. 1) of the reconstructed passages; unused slots -INFINITY
 *   hip_stream  a hipStream_t (NULL = the default stream); the call is asynchronous on it
 * Errors: PLAID_EINVAL for null pointers or out-of-range sizes, PLAID_ENOMEM when the workspace cannot be
 * allocated, PLAID_EHIP for launch failures. */
int plaid_search(plaid_index *idx, const float *Q, int32_t nq, int32_t nprobe, float t_cs, int32_t ndocs,
                 int32_t k, int32_t *out_ids, float *out_scores, void *hip_stream);

/* plaid_search that also copies the intermediates named in *dbg out of the workspace (same kernels, same
 * results).  dbg = NULL behaves like plaid_search. */
int plaid_search_debug(plaid_index *idx, const float *Q, int32_t nq, int32_t nprobe, float t_cs, int32_t ndocs,
                       int32_t k, int32_t *out_ids, float *out_scores, void *hip_stream,
                       const plaid_debug_buffers *dbg);

/* plaid_search for callers that cannot allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc): same arguments, same kernels and bit-identical results, but the workspace is a
 * 64 MiB array inside the library (one copy per device, held until the process ends) instead of memory the library
 * allocates, so the call performs no hipMalloc / hipFree and no other allocating call.  Batches are processed in
 * chunks that fit the array; PLAID_EINVAL when even one query does not fit (plaid_workspace_bytes with nq = 1 tells:
 * about 132 C + 16 P bytes).  Every call on a device uses that device's one array, which keeps the previous call's
 * contents (what must start at zero is cleared by the first kernel of each chunk): calls that overlap on one device
 * race, whichever index they use.  Stage timing and debug outputs are not available through this entry point. */
int plaid_search_static(plaid_index *idx, const float *Q, int32_t nq, int32_t nprobe, float t_cs, int32_t ndocs,
                        int32_t k, int32_t *out_ids, float *out_scores, void *hip_stream);

/* Vanilla ColBERTv2 retrieval, the baseline the paper measures PLAID against (Sections 3.1-3.2, 4.1), on the same index
 * and with the same kernels for Eq. 2, decompression and MaxSim:
 *   1. S_cq and the nprobe best centroids of every query token, as in plaid_search;
 *   2. the inverted list of a centroid holds the ids of the EMBEDDINGS assigned to it; the candidates are the passages
 *      owning an embedding of a probed list (the library builds these lists and a token -> passage map on the first
 *      call: 8 bytes per embedding, kept until plaid_index_free; fewer than 2^31 embeddings);
 *   3. when a query has more than ncandidates candidates they are pruned by scoring the embeddings of the probed lists
 *      -- only those -- with full residual decompression: score = sum over the query tokens of the maximum over the
 *      passage's embeddings among them, the best ncandidates by (score descending, pid ascending) stay;
 *   4. every token of every remaining candidate is decompressed and scored exactly (Eq. 1); the best k are returned
 *      like plaid_search returns them.
 * dbg may be NULL; its pointers are DEVICE, caller-owned and may each be NULL:
 *   cand [nq][P] ascending candidate pids, n_cand [nq];  kept_ids / kept_scores [nq][ncandidates] the candidates after
 *   step 3 in unspecified order with their pruning scores (0 for a query that needed no pruning), n_kept [nq].  Step 3
 *   may decide most candidates by coarse scores and a bound of their error; with kept_scores it scores all of them in
 *   full (the same candidates stay).
 * The first call synchronises the device.  Errors as plaid_search. */
typedef struct {
    int32_t *cand;
    int32_t *n_cand;
    int32_t *kept_ids;
    float *kept_scores;
    int32_t *n_kept;
} plaid_vanilla_debug;
int plaid_search_vanilla(plaid_index *idx, const float *Q, int32_t nq, int32_t nprobe, int32_t ncandidates, int32_t k,
                         int32_t *out_ids, float *out_scores, void *hip_stream, const plaid_vanilla_debug *dbg);

/* Decompress the tokens of n listed passages (Section 4.5: packed byte -> bucket indices through the
 * 256-entry table, value = centroid + bucket weight, one fp32 addition per element).
 *   pids         DEVICE [n] passage ids
 *   out_offsets  DEVICE [n+1] receives the exclusive prefix sum of the passages' token counts (may be NULL)
 *   out_vectors  DEVICE [total][128] fp32 reconstructed vectors, passages concatenated in list order (may be NULL)
 *   out_indices  DEVICE [total][128] uint8 unpacked bucket indices (may be NULL)
 *   capacity     rows available in out_vectors / out_indices; PLAID_EINVAL if total exceeds it
 * Waits for the stream to reach the call (the device checks the ids and reports the total), the first 500 us of it without
 * giving up the processor, and not for the vectors: pids and out_offsets must stay as they are until the stream has passed
 * the call.  A refused list (PLAID_EINVAL: an id outside [0, num_passages), more tokens than capacity) leaves nothing on the
 * stream; out_vectors and out_indices are then untouched, out_offsets too for an id out of range, and hold the prefix sum for a
 * capacity too small.  PLAID_EHIP on a stream that is being captured. */
int plaid_decompress_passages(plaid_index *idx, const int32_t *pids, int32_t n, int64_t *out_offsets,
                              float *out_vectors, uint8_t *out_indices, int64_t capacity, void *hip_stream);

/* Sizes of a loaded index: any pointer may be NULL. */
int plaid_index_info(const plaid_index *idx, int64_t *num_centroids, int64_t *num_passages,
                     int64_t *num_embeddings, int32_t *nbits, int64_t *ivf_len);

/* Which kernel computes S_cq (Eq. 2) for this index: HOST *form =
 *   2  the half-precision matrix instruction on operands split into two fp16 terms each (the default).  Scores are
 *      within 2^-15 of the exact dot products for vectors of norm <= 1 whose components lie in fp16's range (observed:
 *      a few 1e-7); every decision taken on them -- probed centroids (Section 4.1), the pruning map (Eq. 5) -- is
 *      completed in double wherever that bound leaves it open, and the rows of the surviving centroids that stage 2
 *      scores with are re-evaluated in double, so probes, candidates, the pruning map and the stage-2 scores of
 *      queries with at most 63 surviving centroids are those of forms 0 and 1; stage-3 and final scores inherit the
 *      bound (32 entries per score).  Serves nprobe <= 8; a search with a larger nprobe runs form 1 (or 0).  Needs
 *      centroid components below 32 in magnitude: an index whose table exceeds that is given form 1 (or 0) instead.
 *   1  the double-precision matrix instruction, 0  a vector fused-multiply-add chain: both accumulate each score in
 *      double over the dimensions in index order and round once, the definition's bits.  Form 1 is used only when a
 *      check run on the device at the first index creation of the process confirms that the instruction adds its
 *      products in that order.
 * The environment variable PLAID_SCQ_FORM=vector|matrix|split16 (read at index creation) overrides the choice (matrix is
 * an error when the check fails). */
int plaid_get_score_kernel(const plaid_index *idx, int32_t *form);

/* How candidates and their pruned scores (Section 4.1, Eq. 3-5) are computed for this index: HOST *form = 1 or 2 for
 * the inverted form (a passage holds centroid c exactly when c's inverted list holds the passage, so the candidate set
 * and every pruned bag follow from the lists of the probed and the surviving centroids), 0 for the union of the probed
 * lists followed by a stream over the candidates' token codes.  Same results either way.  The inverted form needs a
 * table of num_centroids x (num_passages / R + 1) 32-bit positions, R = 2048 passages per column (form 1) or 8192
 * (form 2), built at index creation with the smaller R whose table is at most 32 MiB or at most four times the size of
 * the inverted lists (device memory of the library's own, beside the index);
 * PLAID_STAGE2_FORM=stream|inverted|inverted11|inverted13 (read at index creation) overrides. */
int plaid_get_stage2_kernel(const plaid_index *idx, int32_t *form);

/* Per-stage GPU time of the most recent plaid_search on this index when stage timing is on
 * (plaid_set_stage_timing(idx, 1)): HOST out_ms[PLAID_NUM_STAGES], summed over the call's query chunks.
 * Turning timing on makes every search synchronise at its end. */
#define PLAID_NUM_STAGES 10
/* stage order: 0 workspace clearing + query layout, 1 S_cq + pruning map (Eq. 2, 5), 2 top-nprobe, probe union and
 * table of surviving centroids, 3 candidate union (Section 4.1), 4 stage-2 interaction (Eq. 3-5), 5 select ndocs,
 * 6 stage-3 interaction (Eq. 3-4), 7 select ndocs/4, 8 stage-4 decompress + MaxSim (Section 4.5, Eq. 1), 9 top-k.  What
 * one kernel does of two stages counts for the later one: with the inverted form 3 is in 4, in short launches the probe union of 2
 * too, and with short lists, few in all, 7 is in 8. */
int plaid_set_stage_timing(plaid_index *idx, int32_t on);
int plaid_get_stage_ms(const plaid_index *idx, float *out_ms);

/* The clock the chip held while the S_cq kernel (Eq. 2; score kernel 2 of plaid_get_score_kernel only) of the most
 * recent plaid_search with stage timing on was running: HOST out_ticks[2] = how far the shader-clock counter
 * (out_ticks[0]) and the fixed-rate 100 MHz timer (out_ticks[1]) moved, each summed over the kernel's workgroups;
 * 100 * out_ticks[0] / out_ticks[1] is the shader clock in MHz.  Both are 0 when nothing was measured.  Synchronises
 * the device.  A diagnostic, like the stage times: the published peak rates assume the chip's top clock. */
int plaid_get_score_kernel_clocks(const plaid_index *idx, uint64_t *out_ticks);

/* Storage variant (Section 4.5 reconstructs the stored embedding and is silent on its length; the embeddings that were
 * stored have unit length, Section 3.1, the reconstruction centroid + residual does not): on != 0 makes every later
 * plaid_search / plaid_search_debug / plaid_search_static on this index score, and plaid_decompress_passages return,
 * reconstructed vectors scaled back to unit length: each token's vector is multiplied by
 * fl32(1 / sqrt(sum of the squares of its fp32 components, added in double in index order)) (0 for a zero vector).
 * The first call with on != 0 computes that factor for every token (num_embeddings floats of device memory owned by the
 * index; the call synchronises the device's default stream); on = 0 switches back.  Stages 1-3 use centroids only and
 * do not change.  Not to be called while a search on this index is in flight.  plaid_search_vanilla returns
 * PLAID_EINVAL while the variant is on.  Errors: PLAID_EINVAL (null index), PLAID_ENOMEM, PLAID_EHIP. */
int plaid_index_set_renormalize(plaid_index *idx, int32_t on);

/* Limit on queries processed per internal chunk (0 = library default).  Affects workspace size only. */
int plaid_set_max_chunk(plaid_index *idx, int32_t max_queries_per_chunk);

/* Bytes of device workspace a plaid_search with these parameters allocates (once, grown on demand, kept until
 * plaid_index_free) on an index with C centroids and P passages, and the number of queries the call processes per
 * internal chunk.  Host arithmetic only: no device is touched.  max_queries_per_chunk as for plaid_set_max_chunk
 * (0 = the library's default: up to 512 queries within about 24 GiB).  bytes: HOST, required; queries_per_chunk: HOST,
 * may be NULL.  Errors: PLAID_EINVAL. */
int plaid_workspace_bytes(int64_t C, int64_t P, int32_t nq, int32_t nprobe, int32_t ndocs, int32_t k,
                          int32_t max_queries_per_chunk, int64_t *bytes, int32_t *queries_per_chunk);

/* ---- Index construction: the step before the search path.  Every array is DEVICE memory of `device`; the calls
 * synchronise `hip_stream` before they return (sizes and error flags are read back) and allocate temporary device
 * memory, which they release. ---- */

/* Nearest centroid of each vector (Section 3.1: a token is stored with the id of its closest centroid):
 * codes[j] = the centroid with the largest dot product centroids[c] . x[j], the dot products accumulated in double over
 * the dimensions in index order and rounded once to fp32, exactly as S_cq of Eq. 2 is (a screening in half
 * precision with a proven error bound decides what it can, these dot products the rest); among equal scores the smaller id wins.
 *   centroids  [C][128] fp32, 16-byte aligned     x  [n][128] fp32, 16-byte aligned     codes  [n] int32 (output)
 * Errors: PLAID_EINVAL (null or misaligned pointers, sizes out of range), PLAID_ENOMEM, PLAID_EHIP. */
int plaid_assign_centroids(const float *centroids, int64_t C, const float *x, int64_t n, int32_t *codes, int device,
                           void *hip_stream);

/* Residual encoding (Section 3.1; the inverse of the byte table of Section 4.5): per dimension r = x - centroid (one
 * fp32 subtraction), bucket = the number of cut-offs strictly below r, and 8 / nbits bucket indices per byte, the first
 * dimension in the most significant bits.
 *   cutoffs    [2^nbits - 1] fp32 ascending        codes  [n] in [0, C)
 *   residuals  [n][16 * nbits] uint8 (output), 4-byte aligned
 * Errors: PLAID_EINVAL (also when a code is outside [0, C): nothing is read out of bounds), PLAID_ENOMEM, PLAID_EHIP. */
int plaid_encode_residuals(const float *centroids, int64_t C, const float *x, const int32_t *codes, int64_t n,
                           const float *cutoffs, int32_t nbits, uint8_t *residuals, int device, void *hip_stream);

/* Passage-level inverted lists (Section 4.1): list c = the ascending unique ids of the passages with a token coded c.
 *   codes        [N] in [0, C)            doc_offsets  [P+1], from 0 to N, non-decreasing
 *   ivf_offsets  [C+1] int64 (output)     ivf_pids     [capacity] int32 (output; NULL: offsets and length only)
 *   ivf_len      HOST, receives ivf_offsets[C] (may be NULL)
 * Errors: PLAID_EINVAL (malformed offsets, a code out of range, capacity below the length), PLAID_ENOMEM, PLAID_EHIP. */
int plaid_build_ivf(const int32_t *codes, const int64_t *doc_offsets, int64_t P, int64_t N, int64_t C, int64_t *ivf_offsets,
                    int32_t *ivf_pids, int64_t capacity, int64_t *ivf_len, int device, void *hip_stream);

/* ---- Reader: what answers from the passages a search has found.  A decoder's layer attends to its own tokens, which a paged
 * cache in four bits a value holds, and to the states of the passages found.  None of these calls needs an index; every array
 * is DEVICE memory of `device`, the calls are asynchronous on `hip_stream`, wait for nothing, allocate nothing and may be
 * captured in a graph.  Offsets and lengths live on the device, so the kernels check them: a value that points outside an
 * array is cut to it (what such a request gets is unspecified, nothing is accessed out of bounds). ---- */

typedef enum { PLAID_BF16 = 0, PLAID_FP16 = 1 } plaid_dtype;

/* Blocks and slots of a step's new tokens.  Request r holds lengths[r] tokens in its first ceil(lengths[r] / block_size) blocks
 * and gets added[r] more (negative numbers count as 0; lengths[r] + added[r] < 2^31).  Blocks are handed out from free_blocks in
 * its order, to request 0 first; a block past its end is -1, a block past max_blocks is neither handed out nor counted.
 *   lengths, added  [n] int32, n >= 1
 *   table           [n][max_blocks] int32, rows table_stride apart; the new entries are written, no other
 *   free_blocks     [n_free] int32 (may be NULL when n_free = 0)
 *   block_size      tokens of a block: 16, 32, 64, 128 or 256
 *   offsets         [n+1] int64 (output) exclusive prefix sum of added
 *   totals          [n] int32 (output) lengths + added
 *   positions       [capacity] int32 (output) place of each new token in its request
 *   slots           [capacity] int64 (output) block * block_size + position % block_size; -1 without a block
 *                   both are -1 from offsets[n] on; tokens past capacity are left out
 *   blocks_wanted   [1] int64 (output) blocks asked for in all: more than n_free means that some are missing
 *   workspace       plaid_block_tables_workspace bytes, 16-byte aligned (may be NULL where that is 0)
 * Errors: PLAID_EINVAL, PLAID_EHIP. */
int plaid_block_tables(const int32_t *lengths, const int32_t *added, int32_t n, int32_t *table, int64_t table_stride,
                       int32_t max_blocks, const int32_t *free_blocks, int32_t n_free, int32_t block_size, int64_t *offsets,
                       int32_t *totals, int32_t *positions, int64_t *slots, int64_t capacity, int64_t *blocks_wanted,
                       void *workspace, int64_t workspace_bytes, int device, void *hip_stream);
int plaid_block_tables_workspace(int32_t n, int64_t capacity, int64_t *bytes);

/* A paged cache of keys and values in four bits a value.  Every 32 dimensions of a token's head share a power of two, stored
 * as its biased exponent (255: the group holds a value that is not finite, all of it reads as NaN); a value is a sign and one
 * of 0 0.5 1 1.5 2 3 4 6 (codes 0-7, the sign is bit 3) times that power.  data: [num_blocks][kv_heads] regions of
 * block_size * head_dim * 17 / 16 bytes: the codes of the keys, the codes of the values, the scales of the keys, the scales of
 * the values.  Key codes [token][head_dim / 2], the even dimension in the low half of a byte; value codes in cells of 16 tokens
 * [token / 16][token / 4 % 4][dim % 16][dim / 32][token % 4], the halves of a byte being dimensions 32 i + m and
 * 32 i + 16 + m; scales [token][head_dim / 32].  dtype is the type of what is written, and what it is read as. */
typedef struct {
    uint8_t *data; /* 16-byte aligned */
    int64_t num_blocks;
    int32_t block_size; /* 16, 32, 64, 128 or 256 */
    int32_t kv_heads;
    int32_t head_dim; /* 64 or 128 */
    int32_t dtype;    /* plaid_dtype */
} plaid_paged_cache;

/* Writes keys and values of n tokens (k, v: rows token_stride apart, heads head_stride, in elements, multiples of 8 in [0, 2^24);
 * 16-byte aligned) to their slots; a slot outside [0, num_blocks * block_size) is left out, two equal slots are a caller's
 * mistake.  The power of two of a group is the smallest that keeps its largest magnitude within 6 (bf16: 2^-126 .. 2^126,
 * fp16: 2^-23 .. 2^14), values round to the nearest code, ties to the even one, and stay finite in the type. */
int plaid_cache_write(const plaid_paged_cache *cache, const void *k, const void *v, int64_t k_token_stride,
                      int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots, int64_t n,
                      int device, void *hip_stream);
/* The keys and values that n slots hold, k and v [n][kv_heads][head_dim] contiguous (either may be NULL); zero for a slot
 * outside the cache.  Exact: every code is a value of the type. */
int plaid_cache_read(const plaid_paged_cache *cache, const int64_t *slots, int64_t n, void *k, void *v, int device,
                     void *hip_stream);

/* Arguments of an attention call.  Row (token i of request r, head h) attends with key head h * kv_heads / heads:
 *   s_j = scale * q . k_j + key_bias_j,   out = sum_j softmax(s)_j v_j,   lse = log sum_j exp(s_j);
 * a row that no key is left for gives zeros and -INFINITY.  lse is two numbers to be added, a shift
 * (0 unless the largest of a request's biases is above 256, or below -256) and the rest, so that it is whole where all scores are as low as
 * the type goes.  Sums, softmax statistics and their exponentials are held in 32
 * bits; the softmax's weights round to the type before they multiply the values.
 *   q, k, v          [num_queries | num_keys][heads | kv_heads][head_dim] of dtype, 16-byte aligned, the strides of tokens and
 *                    heads in elements, multiples of 8 in [0, 2^24); k and v are those of plaid_cross_attention
 *   key_bias         [num_keys] of dtype, or NULL; a key of bias -INFINITY takes no part, whatever k and v hold there
 *   q_offsets        [n+1] int64: the tokens of request r are rows q_offsets[r] .. q_offsets[r+1]-1; rows outside every request
 *                    are not written
 *   k_offsets        [n+1] int64, the same for the keys (plaid_cross_attention)
 *   out              [num_queries][heads][head_dim] contiguous, lse [num_queries][heads][2] fp32 or NULL
 * heads is a multiple of kv_heads, head_dim 64 or 128; num_queries * (heads / kv_heads)^2 < 2^32.  A scale may be negative.
 * What a key holds reaches the rows that see it, and no other, also where it is not finite. */
typedef struct {
    int32_t dtype;
    int32_t n;
    int32_t heads;
    int32_t kv_heads;
    int32_t head_dim;
    float scale;
    int64_t num_queries;
    int64_t num_keys;
    const void *q;
    const void *k;
    const void *v;
    const void *key_bias;
    int64_t q_token_stride;
    int64_t q_head_stride;
    int64_t k_token_stride;
    int64_t k_head_stride;
    int64_t v_token_stride;
    int64_t v_head_stride;
    const int64_t *q_offsets;
    const int64_t *k_offsets;
    void *out;
    float *lse;
} plaid_attention;

/* Attention over a paged cache.  Request r's keys are the lengths[r] tokens that its row of `table` ([n][max_blocks] int32, rows
 * table_stride apart) leads to; a block id outside the cache hides its tokens.  causal != 0: the request's queries are its last
 * tokens, in order, and query i of m sees the first lengths[r] - m + i + 1.  k, v, key_bias, num_keys and k_offsets of *args are
 * not looked at; kv_heads, head_dim and dtype are the cache's.
 * workspace: plaid_cached_attention_workspace bytes, 16-byte aligned. */
int plaid_cached_attention(const plaid_attention *args, const plaid_paged_cache *cache, const int32_t *table,
                           int64_t table_stride, int32_t max_blocks, const int32_t *lengths, int32_t causal, void *workspace,
                           int64_t workspace_bytes, int device, void *hip_stream);
int plaid_cached_attention_workspace(const plaid_attention *args, int32_t max_blocks, int32_t block_size, int64_t *bytes);

/* Attention to states of another length (an encoder's, or those of the passages found: plaid_decompress_passages' offsets are
 * k_offsets, taken once a request).  workspace: plaid_cross_attention_workspace bytes (backward = 0), 16-byte aligned. */
int plaid_cross_attention(const plaid_attention *args, void *workspace, int64_t workspace_bytes, int device, void *hip_stream);
/* Its gradients: with P = exp(s - lse), dP = d_out . v and dS = P (dP - d_out . out),
 *   dv_j = sum P d_out,  dk_j = scale sum dS q,  dq_i = scale sum_j dS k,  dbias_j = sum of dS over all rows and heads.
 * args->out and args->lse are what the forward call gave; d_out [num_queries][heads][head_dim] contiguous; dq like d_out, dk and
 * dv [num_keys][kv_heads][head_dim] contiguous, dbias [num_keys], all of dtype; each may be NULL, which changes nothing of the others.  Every
 * sum has one order: the same inputs give the same bits.  dq, dk and dbias are zero where one key of a request can have a weight.  fp16: the
 * gradient's range is the type's, so the caller scales the loss. */
int plaid_cross_attention_backward(const plaid_attention *args, const void *d_out, void *dq, void *dk, void *dv, void *dbias,
                                   void *workspace, int64_t workspace_bytes, int device, void *hip_stream);
int plaid_cross_attention_workspace(const plaid_attention *args, int32_t backward, int64_t *bytes);

/* ---- Training a reader: what a training step does around its attention -- tokens in, states between the layers, states into a loss.
 * The rules of the reader's calls hold: no index, arrays of `device`, asynchronous on `hip_stream`, nothing waited for or allocated, and a
 * call may be captured in a graph.  dtype is a plaid_dtype, that of all states, parameters and their gradients; results are formed in
 * 32 bits and rounded once.  Every sum has one order: the same inputs give the same bits.  Strides are in elements, from one row to
 * the next; outputs are contiguous.  Outputs overlap no input, but where it says so. ---- */

/* Rows of a table for n tokens: out[t] = scale * table[ids[t]]; zeros for an id outside [0, vocabulary).
 *   table  [vocabulary][width], table_stride apart     ids  [n] int64     out  [n][width], 16-byte aligned
 * width 1 .. 2^20, n and vocabulary up to 2^30, n * width and vocabulary * width up to 2^40. */
int plaid_embedding(const void *table, int64_t table_stride, int64_t vocabulary, int32_t width, const int64_t *ids, int64_t n,
                    float scale, void *out, int32_t dtype, int device, void *hip_stream);
/* The table's gradient: d_table[v] = scale * the sum of d_out[t] over the tokens t of id v, zeros where there is none; with add != 0 the
 * sum is added to what d_table holds, and rows without a token stay as they are (a table that is used twice, or that is the loss's
 * vocabulary too).  A token of an id outside [0, vocabulary) is not read.
 *   d_out  [n][width], d_out_stride apart     d_table  [vocabulary][width]
 * workspace: plaid_embedding_backward_workspace bytes, 16-byte aligned. */
int plaid_embedding_backward(const void *d_out, int64_t d_out_stride, int64_t vocabulary, int32_t width, const int64_t *ids, int64_t n,
                             float scale, int32_t add, void *d_table, int32_t dtype, void *workspace, int64_t workspace_bytes,
                             int device, void *hip_stream);
int plaid_embedding_backward_workspace(int64_t n, int64_t vocabulary, int32_t width, int64_t *bytes);

/* Dropout, with a residual added: out[e] = residual[e] + (kept ? x[e] / (1 - T / 65536) : 0), T = p * 65536 rounded to a whole number
 * (halves up), for elements e = 0 .. n-1 in memory's order.  The mask is never stored: element e is kept where 16 bits of
 * Philox4x32-10 are at least T -- key: rng[0], counter: e / 8 (low half first) and rng[1]; of its four words, element e takes word
 * e / 2 % 4, the low half where e is even.  The gradient of x is the same call on d_out without a residual, that of the residual is d_out.
 *   x, residual  [n] (residual may be NULL)     rng  [2] int64 on the device: a seed, and a number that each call of a program's has for
 *   itself     out  [n]; may be x or residual
 * p in [0, 1] (1: nothing is kept), n up to 2^40. */
int plaid_dropout(const void *x, const void *residual, int64_t n, float p, const int64_t *rng, void *out, int32_t dtype, int device,
                  void *hip_stream);

/* Layer norm of rows: with m a row's mean and r = 1 / sqrt(its variance + eps), out = (x - m) r weight + bias.
 *   x  [rows][width], x_stride apart     weight, bias  [width], each may be NULL     out  [rows][width]
 *   statistics  [rows][2] fp32 (output, may be NULL) m and r, for the backward pass
 * width 1 .. 16384, eps not negative. */
int plaid_layer_norm(const void *x, int64_t x_stride, const void *weight, const void *bias, int64_t rows, int32_t width, float eps,
                     void *out, float *statistics, int32_t dtype, int device, void *hip_stream);
/* Its gradients: with x^ = (x - m) r and g = d_out weight, dx = r (g - mean g - x^ mean (g x^)), dweight = sum over rows of d_out x^,
 * dbias = sum over rows of d_out.  dx, dweight and dbias may each be NULL; dweight takes a weight.
 * workspace: plaid_layer_norm_backward_workspace bytes, 16-byte aligned (not looked at without dweight and dbias). */
int plaid_layer_norm_backward(const void *d_out, int64_t d_out_stride, const void *x, int64_t x_stride, const void *weight,
                              const float *statistics, int64_t rows, int32_t width, void *dx, void *dweight, void *dbias, int32_t dtype,
                              void *workspace, int64_t workspace_bytes, int device, void *hip_stream);
int plaid_layer_norm_backward_workspace(int64_t rows, int32_t width, int64_t *bytes);

/* Softmax cross entropy of states over a vocabulary, without the scores in memory: with s_tv = scale * hidden[t] . weight[v],
 *   lse[t] = log sum_v exp(s_tv),   loss[t] = lse[t] - s_t,targets[t].
 * A row whose target is outside [0, vocabulary) takes no part: its loss is 0, its gradient zero, and what it holds reaches nothing.
 *   hidden   [rows][width], weight  [vocabulary][width]: 16-byte aligned, strides multiples of 8 in [0, 2^24)
 *   targets  [rows] int64
 *   loss     [rows] fp32     lse  [rows][2] fp32 or NULL: two numbers to be added, the largest score and the rest
 * width a multiple of 8 up to 16384, rows up to 2^24, vocabulary up to 2^27. */
typedef struct {
    int32_t dtype;
    int32_t width;
    int64_t rows;
    int64_t vocabulary;
    float scale;
    const void *hidden;
    const void *weight;
    int64_t hidden_stride;
    int64_t weight_stride;
    const int64_t *targets;
    float *loss;
    float *lse;
} plaid_token_loss;

/* workspace: plaid_cross_entropy_workspace bytes (backward = 0 or 1), 16-byte aligned. */
int plaid_cross_entropy(const plaid_token_loss *args, void *workspace, int64_t workspace_bytes, int device, void *hip_stream);
/* Its gradients, the scores formed again over a piece of the vocabulary at a time: with G_tv = d_loss[t] (exp(s_tv - lse[t]) - [v = target]),
 *   d_hidden[t] = scale sum_v G_tv weight[v],   d_weight[v] = scale sum_t G_tv hidden[t]   (contiguous, either may be NULL).
 * args->lse is what the forward call gave, args->loss is not looked at.  d_loss [rows] fp32, d_loss_stride 1, or 0: one number for all rows.
 * G rounds to the type before it is multiplied, in fp16 in steps of 2^-39 of the power of two above d_loss or more (what its targets' entries
 * lose by that is multiplied too); that power is kept apart from it.  For d_weight the states carry it and round to the type: what is lost of
 * a row's is 2^-126 of the largest d_loss in bf16, 2^-40 of the largest product of a state and its row's d_loss in fp16.  lse keeps a row's
 * largest score in 32 bits: where scores are far from zero, probabilities are off by 2^-24 of it, relative. */
int plaid_cross_entropy_backward(const plaid_token_loss *args, const float *d_loss, int64_t d_loss_stride, void *d_hidden, void *d_weight,
                                 void *workspace, int64_t workspace_bytes, int device, void *hip_stream);
int plaid_cross_entropy_workspace(const plaid_token_loss *args, int32_t backward, int64_t *bytes);

/* Thread-local message describing the most recent error on the calling thread ("" if none). */
const char *plaid_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* PLAID_H */
