/*
 * ivfpq.h -- C ABI of the MI355X (gfx950) IVFPQ search library.
 *
 * The library implements the search phase of IVFPQ as described in
 * arXiv 2301.06672, Sec. I-C (second enumeration) and Sec. I-D, with the
 * "norm2 fragment lookup table" held in LDS as fp32, IEEE half or one of the
 * paper's sign-less 8-bit floats, e5m3 and e4m4 (Sec. II).  All compute of the search runs in
 * hand-written HIP kernels; this header is the only interface.
 *
 * Conventions
 *  - Every function returns an ivfpq_status (0 = OK, negative = error); nothing
 *    throws across the ABI.  ivfpq_last_error() gives a text for the last
 *    non-OK return on the calling thread.
 *  - "host" pointers are ordinary CPU memory, "device" pointers are HIP device
 *    memory of the current device.  The caller owns every buffer it passes; the
 *    library never allocates or frees device memory.
 *  - Row-major everywhere.  Distances are squared L2 (Sec. I-B).
 *  - hip_stream is a hipStream_t passed as void* (NULL = the default stream).
 *    Search calls only enqueue work; they do not synchronise.
 *  - The library reads no environment variable; launch heuristics can be overridden per index with
 *    ivfpq_set_tuning (for tuning experiments and tests only).
 *  - No function throws: a C++ exception inside the library (host memory exhausted) comes back as a status.
 */
#ifndef IVFPQ_H
#define IVFPQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ivfpq_index ivfpq_index_t; /* opaque; created by build/import, destroyed by ivfpq_free */

/* Storage type of the lookup-table entries F(y_v) in LDS (Sec. I-D, Sec. II). */
typedef enum {
    IVFPQ_LUT_FP32 = 0,     /* IEEE binary32 */
    IVFPQ_LUT_FP16 = 1,     /* IEEE binary16, round-to-nearest-even, saturating at 65504 */
    IVFPQ_LUT_FP8_E5M3 = 2, /* 5 exponent + 3 mantissa bits, no sign, bias 15, all codes normal:
                               value(b) = (1 + (b&7)/8) * 2^((b>>3) - 15); FP32 -> code: nearest, ties up,
                               clamped to [0x00, 0xFF]; code -> FP32 bits: (b << 20) + 0x38000000 */
    IVFPQ_LUT_FP8_E4M4 = 3  /* the paper's other split, 4 exponent + 4 mantissa bits, same rules:
                               value(b) = (1 + (b&15)/16) * 2^((b>>4) - bias), 16 binades from 2^-bias;
                               the bias is set per index with ivfpq_set_e4m4_bias (default 7) */
} ivfpq_lut_dtype_t;

/* Rounding of the FP32 -> 8-bit encode (Sec. II: "shift the bit string and adjust the exponent bias";
 * whether the shift rounds is left open by the text). */
typedef enum {
    IVFPQ_ROUND_NEAREST = 0, /* nearest representable value, ties to the larger one (the default) */
    IVFPQ_ROUND_TRUNCATE = 1 /* the largest representable value not above the input: a bare shift */
} ivfpq_fp8_rounding_t;

typedef enum {
    IVFPQ_OK = 0,
    IVFPQ_EINVAL = -1,       /* null pointer, bad shape or parameter */
    IVFPQ_ENOSPACE = -2,     /* a caller buffer is smaller than the matching *_bytes() query says */
    IVFPQ_EHIP = -3,         /* a HIP runtime call failed (text in ivfpq_last_error) */
    IVFPQ_EUNSUPPORTED = -4, /* shape outside what the kernels handle (e.g. table does not fit LDS) */
    IVFPQ_ESTATE = -5        /* index not uploaded, or uploaded to another device */
} ivfpq_status;

enum { IVFPQ_MAX_K = 1024, IVFPQ_MAX_PROBES = 1024 };

/* ---- index construction (Sec. I-C, first enumeration; host side, not timed) ---- */

/* Builds an index on the host CPU: (1) Lloyd k-means with n_lists clusters (kmeans_iters
 * iterations, start rows drawn from `seed`), (2) residuals to the own centroid, (3) product
 * quantisation of the residuals: pq_dim contiguous sub-vectors of d/pq_dim components, one
 * codebook of 2^pq_bits entries per sub-space, (4) the saved lists, codes and codebook.
 * data: host [n][d] fp32.  Requires d % pq_dim == 0, 4 <= pq_bits <= 8 (the paper treats 8),
 * (pq_dim*pq_bits/8) % 4 == 0, 1 <= n_lists <= n.  *out receives the new handle. */
int ivfpq_build_host(const float* data, int64_t n, int32_t d, int32_t n_lists, int32_t pq_dim,
                     int32_t pq_bits, int32_t kmeans_iters, uint64_t seed, ivfpq_index_t** out);

/* The same four build steps on the GPU (current device).  d_data: device [n][d] fp32, n < 2^31.
 * Every decision (nearest cluster centre, nearest codeword) is the arg-min of float64 squared
 * distances, ties to the lower index; every centre is the float64 mean of its members summed in
 * ascending row order, rounded to fp32 once; an empty cluster keeps its centre.
 * The random draws are inputs (host arrays; each may be NULL, then it is drawn from `seed` as
 * ivfpq_build_host does):
 *   coarse_train_rows [n_coarse_train]  rows of d_data the cluster k-means trains on
 *                                       (NULL: <= 256 rows per list at a fixed stride)
 *   coarse_init_rows  [n_lists]         positions in that training set whose rows start the k-means
 *   pq_train_rows     [n_pq_train]      rows of d_data whose residuals train the codebooks
 *                                       (NULL: <= 262144 rows at a fixed stride); n_pq_train * pq_dim < 2^32
 *   pq_init_rows      [pq_dim][2^pq_bits]  positions in that training set, per sub-space
 * d_workspace: device scratch of >= ivfpq_build_device_workspace_bytes(...) (pass the two counts, or 0
 * for the defaults), 256-byte aligned.  Synchronises the stream before it returns; the resulting handle
 * holds the logical arrays on the host, as after ivfpq_build_host (call ivfpq_upload next). */
size_t ivfpq_build_device_workspace_bytes(int64_t n, int32_t d, int32_t n_lists, int32_t pq_dim, int32_t pq_bits,
                                          int64_t n_coarse_train, int64_t n_pq_train);
int ivfpq_build_device(const float* d_data, int64_t n, int32_t d, int32_t n_lists, int32_t pq_dim, int32_t pq_bits,
                       int32_t kmeans_iters, const int64_t* coarse_train_rows, int64_t n_coarse_train,
                       const int64_t* coarse_init_rows, const int64_t* pq_train_rows, int64_t n_pq_train,
                       const int64_t* pq_init_rows, uint64_t seed, void* d_workspace, size_t workspace_bytes,
                       void* hip_stream, ivfpq_index_t** out);

/* Build step 1's assignment alone, for inspection: d_labels[i] (device, int32) = the centre nearest to
 * row i of d_rows (device [n_rows][d]) among d_centres (device [n_centres][d]), decided as above.
 * d_workspace >= ivfpq_assign_device_workspace_bytes(n_rows, d, n_centres).  Asynchronous. */
size_t ivfpq_assign_device_workspace_bytes(int64_t n_rows, int32_t d, int32_t n_centres);
int ivfpq_assign_device(const float* d_rows, int64_t n_rows, int32_t d, const float* d_centres, int32_t n_centres,
                        int32_t* d_labels, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Imports the logical saved index (Sec. I-C build step 4).  All host pointers; the library copies.
 *   centroids    [n_lists][d] f32
 *   codebooks    [pq_dim][2^pq_bits][d/pq_dim] f32
 *   list_offsets [n_lists+1] i64, non-decreasing, [0] = 0, [n_lists] = n
 *   codes        [n][pq_dim*pq_bits/8] u8 in list order: the codes of a vector are one string of
 *                pq_dim*pq_bits bits, sub-space j in bits [j*p, (j+1)*p), bit i of the string = bit
 *                (i mod 8) of byte (i div 8).  pq_bits = 8: byte j = code of sub-space j; pq_bits = 4:
 *                byte j holds sub-space 2j in its low and 2j+1 in its high nibble
 *   ids          [n] i64 in list order (the caller's labels; returned by search) */
int ivfpq_index_from_arrays(int64_t n, int32_t d, int32_t n_lists, int32_t pq_dim, int32_t pq_bits,
                            const float* centroids, const float* codebooks, const int64_t* list_offsets,
                            const uint8_t* codes, const int64_t* ids, ivfpq_index_t** out);

/* Shape of an index; any out pointer may be NULL. */
int ivfpq_index_info(const ivfpq_index_t* index, int64_t* n, int32_t* d, int32_t* n_lists,
                     int32_t* pq_dim, int32_t* pq_bits);

/* Copies the logical arrays (same layout as ivfpq_index_from_arrays) into caller host buffers of
 * the sizes ivfpq_index_info implies; any pointer may be NULL to skip that array. */
int ivfpq_index_export(const ivfpq_index_t* index, float* centroids, float* codebooks,
                       int64_t* list_offsets, uint8_t* codes, int64_t* ids);

/* Encoding of one of the two 8-bit table dtypes (lut_dtype = IVFPQ_LUT_FP8_E5M3 or _E4M4) for searches
 * on this index; takes effect at the next call.  Defaults: bias 15 (e5m3) / 7 (e4m4), nearest, fixed.
 *   bias            exponent bias B of the format: value(b) = (1 + mant/2^M) * 2^(exp - B).  Moving the
 *                   bias by s is a scale of the table by 2^s before the encode and 2^-s after the
 *                   decode; returned distances are always in the data's own units.
 *                   -96 <= B <= 110 (e5m3), -100 <= B <= 110 (e4m4): every code a normal FP32 number.
 *   rounding        an ivfpq_fp8_rounding_t
 *   per_table_bias  0: `bias` for every table.  1: per (query, cluster) table, the bias that puts the
 *                   binade of the table's largest entry on the format's top binade (with e the FP32
 *                   exponent of that entry, B = 31 - e for e5m3, 15 - e for e4m4, clamped to the range
 *                   above); `bias` is ignored.  Costs a second pass over the table's entries. */
int ivfpq_set_fp8_encoding(ivfpq_index_t* index, int32_t lut_dtype, int32_t bias, int32_t rounding,
                           int32_t per_table_bias);

/* Shorthand: sets only the exponent bias of the IVFPQ_LUT_FP8_E4M4 table dtype for searches on this index (Sec. II gives the
 * 4+4 split but not its bias): representable table values are 2^-bias .. 1.9375 * 2^(15-bias); what
 * falls outside is clamped to the nearest end.  -100 <= bias <= 110.  Takes effect at the next call. */
int ivfpq_set_e4m4_bias(ivfpq_index_t* index, int32_t bias);

void ivfpq_free(ivfpq_index_t* index);

/* ---- device residency ---- */

/* Bytes of device memory the uploaded index needs (lists are padded to 64 vectors and the codes
 * re-laid out for coalesced wave64 loads; see ivfpq_upload). */
size_t ivfpq_device_bytes(const ivfpq_index_t* index);

/* Writes the device image of the index into d_buf (device, >= ivfpq_device_bytes, 256-byte aligned)
 * on the current device and remembers the pointer.  Synchronous.  d_buf must stay alive and
 * unmodified while the handle is used for searches. */
int ivfpq_upload(ivfpq_index_t* index, void* d_buf, size_t bytes, void* hip_stream);

/* Bytes of device scratch one search call needs for these parameters (probe lists, per-pair
 * descriptors, cluster ranking values, the R rows and the positions of filtered candidates).
 * Large batches are processed in query tiles so that the figure stays within the index's workspace
 * limit (one query's share can exceed it: a tile holds at least one query).  A smaller batch never needs more. */
size_t ivfpq_search_workspace_bytes(const ivfpq_index_t* index, int64_t nq, int32_t n_probes,
                                    int32_t k, int32_t lut_dtype);

/* Overrides one launch heuristic of searches on this index (tuning experiments, tests); value 0 restores
 * the library's own choice.  No knob changes any result.  Takes effect at the next call. */
typedef enum {
    IVFPQ_TUNE_SCAN_THREADS = 0, /* workgroup size of the scan kernels: 64, 128, 256, 512 or 1024 */
    IVFPQ_TUNE_ORDER_BLOCK = 1,  /* consecutive (query, probe) pairs of the cluster-grouped order that stay on one
                                    XCD (>= 1; the scan that shares a workgroup between pairs needs an even value) */
    IVFPQ_TUNE_SCAN_SHARE = 2,   /* 1: one (query, probe) pair per scan workgroup; 2 or 4: up to that many pairs of
                                    one cluster per workgroup wherever the kernel for it applies */
    IVFPQ_TUNE_EARLY_EXIT = 3,   /* 1: on (the default: large batches add up only the vectors that a matrix product
                                    finds able to be among the results; in the table kernels a 64-vector group stops
                                    adding once all its partial sums are over the query's bound); -1: off, every lookup
                                    of Eq. (1) is made.  Leaves the route (SCAN_ROUTE) as it is */
    IVFPQ_TUNE_LDS_PAD = 4,      /* extra bytes of LDS requested per scan workgroup (lowers occupancy without
                                    changing the table: separates the two effects of a smaller table dtype) */
    IVFPQ_TUNE_SCAN_ROUTE = 5    /* how the probes of a query are scanned; the library chooses by the amount of work.
                                    1: all of them in one launch, no filter (small searches); 2: the nearest one
                                    first, the others filtered, query by query; 3: the same with the pairs grouped
                                    by cluster (large batches; implied by a non-zero SCAN_SHARE or ORDER_BLOCK) */
} ivfpq_tuning_t;
int ivfpq_set_tuning(ivfpq_index_t* index, int32_t knob, int32_t value);

/* The workspace limit of searches on this index, in bytes (default 32 GiB; at least 1 MiB).  A query's
 * share of the scratch is sized for the worst case (every vector of its n_probes largest clusters kept),
 * so big indexes split a batch into tiles; fewer, larger tiles run faster (measured: 10,000 queries on
 * 10^8 vectors take 15.3 ms with 2 GiB, 14.0 ms with 8 GiB, 13.5 ms with 32 GiB), smaller limits suit
 * many concurrent callers.  Takes effect at the next ivfpq_search_workspace_bytes / search call. */
int ivfpq_set_workspace_limit(ivfpq_index_t* index, size_t bytes);

/* ---- search (Sec. I-C, second enumeration, steps 1-5) ---- */

/* For each of nq queries: picks the n_probes clusters with the nearest centroids (step 1), and for
 * each picked cluster forms the query residual (step 2), builds the lookup table F in LDS in
 * lut_dtype (step 3), accumulates R = sum_j F(y_j) (Eq. 1) over every coded vector of the cluster
 * (step 4); then keeps the k smallest R over all picked clusters (step 5).
 *   d_queries [nq][d] f32 (device)          d_ids [nq][k] i64 (device, out)
 *   d_dists   [nq][k] f32 (device, out): R of the returned vectors, ascending; ties ordered by id.
 * Rows with fewer than k candidates are padded with id -1, distance +inf.
 * 1 <= n_probes <= min(n_lists, IVFPQ_MAX_PROBES), 1 <= k <= IVFPQ_MAX_K.
 * d_workspace: device scratch of >= ivfpq_search_workspace_bytes(...), 256-byte aligned; calls that
 * may overlap in time need distinct workspaces. */
int ivfpq_search(const ivfpq_index_t* index, const float* d_queries, int64_t nq, int32_t n_probes,
                 int32_t k, int32_t lut_dtype, int64_t* d_ids, float* d_dists,
                 void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ivfpq_search for callers that cannot allocate device memory or provide a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, results and kernels as
 * ivfpq_search, but the scratch is a fixed array of IVFPQ_STATIC_SCRATCH_BYTES inside the library's device
 * image (each GPU the library runs on holds it until the process ends); the call allocates and frees nothing.
 * A batch is processed in as many query tiles as the array requires; if a single query's share does not fit
 * (its n_probes largest clusters hold too many vectors) the call returns IVFPQ_ENOSPACE and touches nothing.
 * All calls on one GPU share that GPU's array, whatever the index or stream: calls that overlap in time race,
 * so issue them on one stream or order them yourself.  Nothing in the array needs to survive between calls. */
#define IVFPQ_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
int ivfpq_search_static(const ivfpq_index_t* index, const float* d_queries, int64_t nq, int32_t n_probes,
                        int32_t k, int32_t lut_dtype, int64_t* d_ids, float* d_dists, void* hip_stream);

/* Step 1 alone: d_probes [nq][n_probes] u32 (device, out), nearest first, ties to the lower
 * cluster index; d_probe_dists [nq][n_probes] f32 (device, out, may be NULL). */
int ivfpq_select_probes(const ivfpq_index_t* index, const float* d_queries, int64_t nq,
                        int32_t n_probes, uint32_t* d_probes, float* d_probe_dists,
                        void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Steps 2-5 on caller-chosen clusters: d_probes [nq][n_probes] u32 (device, in), every entry
 * < n_lists; a cluster listed twice for one query is scanned twice. */
int ivfpq_search_with_probes(const ivfpq_index_t* index, const float* d_queries, int64_t nq,
                             const uint32_t* d_probes, int32_t n_probes, int32_t k, int32_t lut_dtype,
                             int64_t* d_ids, float* d_dists,
                             void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Steps 2-3 alone, for inspection: builds the table of one (query, cluster) pair exactly as the
 * search kernel stages it in LDS and copies the raw bytes out.
 * d_query [d] f32 (device); d_lut_out (device) [pq_dim][2^pq_bits] entries of lut_dtype,
 * i.e. pq_dim * 2^pq_bits * {4, 2, 1, 1} bytes for the four dtypes. */
int ivfpq_dump_lut(const ivfpq_index_t* index, const float* d_query, uint32_t list_id,
                   int32_t lut_dtype, void* d_lut_out, void* hip_stream);

/* Step 4 alone, for inspection: R of every coded vector of one cluster for one query, in list
 * order.  d_R_out (device) [list length] f32. */
int ivfpq_scan_list(const ivfpq_index_t* index, const float* d_query, uint32_t list_id,
                    int32_t lut_dtype, float* d_R_out, void* hip_stream);

/* ---- re-ranking with the stored vectors (not part of the paper's path; the usual companion of a PQ
 * search, whose Eq. (1) only approximates |q - x|^2) ---- */

/* For each of nq queries: the exact squared distance (fp32, direct form) to each of its n_cand candidate
 * vectors, and the k smallest, ascending, ties ordered by id.  A candidate id is a row of d_data
 * (device [n_data][d] fp32: the vectors the index was built from, when their ids are their row numbers);
 * ids outside [0, n_data) -- the -1 padding of a search result -- are skipped; an id listed twice is
 * ranked twice.  d_cand_ids [nq][n_cand] i64 (device), e.g. the ids of ivfpq_search with a larger k.
 * d_ids [nq][k] i64, d_dists [nq][k] f32 (device, out); short rows are padded with -1 / +inf.
 * 1 <= n_cand <= IVFPQ_MAX_K, 1 <= k <= IVFPQ_MAX_K.  Asynchronous; needs no workspace. */
int ivfpq_refine(const float* d_data, int64_t n_data, int32_t d, const float* d_queries, int64_t nq,
                 const int64_t* d_cand_ids, int32_t n_cand, int32_t k, int64_t* d_ids, float* d_dists,
                 void* hip_stream);

/* ---- language models around a search: 8-bit products, neighbours' tokens, log-probabilities, distillation ----
 *
 * A search over hidden states finds the stored states nearest to a query, and each carries the token that followed it.
 * These calls give the model's logits (a product of 8-bit rows), turn search results into a distribution over tokens,
 * score tokens under the model's distribution or its mixture with the neighbours', and train a model towards a few
 * listed tokens (the neighbours', or a teacher model's best).  None needs an index.
 *
 *  - Matrices have rows of contiguous values, `stride` values (not bytes) from one row to the next; pointers and
 *    strides need the alignment of a value only, unless stated.  `dtype` is an ivfpq_values_dtype_t.  Logits and 16-bit
 *    rows are widened to fp32; sums, maxima and statistics are fp32; a result in 16 bits is rounded once, to nearest.
 *  - A call takes up to 2^21 rows of logits of up to 2^30 tokens.
 *  - A token is an int32 in [0, vocab); any other value marks an unused place.
 *  - With T = temperature, 1e-6 <= T <= 1e6, a row of logits x has the distribution p_v = exp((x_v - M)/T) / sum_u exp((x_u - M)/T),
 *    M its largest logit.  A logit of -inf has p = 0; a logit of the type's lowest value is a number like any other.  A row
 *    whose logits are all -inf has no distribution: p = 0 everywhere, entropy 0, gradient 0.  A row that holds a NaN or +inf
 *    has NaN statistics, log-probabilities, losses and gradients.
 *  - norms [n][2] fp32 of a row: M and log(sum_u exp((x_u - M)/T)); {-inf, -inf} of a row without a distribution.
 *    What a backward call needs of the forward pass.
 *  - Calls only enqueue work on hip_stream; a call for zero rows does nothing.  Results do not depend on timing: the
 *    same inputs give the same bits.  Outputs must not overlap inputs, but a gradient may be written over its logits
 *    (same pointer, dtype and stride). */
typedef enum {
    IVFPQ_VALUES_FP32 = 0,
    IVFPQ_VALUES_FP16 = 1, /* IEEE binary16 */
    IVFPQ_VALUES_BF16 = 2  /* the upper half of a binary32 */
} ivfpq_values_dtype_t;

enum {
    IVFPQ_MAX_TOP = 128,     /* alternatives of ivfpq_token_logprobs */
    IVFPQ_MAX_LISTED = 1024, /* listed tokens (neighbours, a teacher's) of a row */
    IVFPQ_MAX_MIXED = 256,   /* alternatives and neighbours together, where both are asked for */
    IVFPQ_MAX_Q8_K = 65536   /* components of an 8-bit row: sums of products stay within int32 */
};

/* Rows as signed 8-bit codes with a scale each: s = max_j |x_j| / 127 in fp32, code_j = x_j / s rounded to the nearest
 * integer (ties to even), within [-127, 127]; s and the codes of a row of zeros are 0.  A row that holds a NaN or an
 * infinity has s = NaN and codes 0.  d_rows [n][d]; d_codes [n][code_stride] int8, of which the codes [d, code_stride) of a
 * row are written as 0, code_stride >= d; d_scales [n] fp32.  1 <= d <= IVFPQ_MAX_Q8_K. */
int ivfpq_quantize_rows(const void* d_rows, int32_t dtype, int64_t n, int32_t d, int64_t row_stride, int8_t* d_codes,
                        int64_t code_stride, float* d_scales, void* hip_stream);

/* out[i][j] = (a_scale[i] * b_scale[j]) * sum_c a[i][c] b[j][c] + bias[j]: the product of 8-bit rows on the matrix cores,
 * summed exactly in int32.  Hidden states (a) and an output embedding (b) give logits; queries and stored vectors give
 * inner products, and with bias[j] = -|b_j|^2 / 2 the largest value of a row is its nearest stored vector.
 *   d_a [m][k], d_b [n][k] int8: both pointers 16-byte aligned, both strides multiples of 16 and at least k rounded up to
 *   16 (at most 2^24); every row's bytes up to there, the last row's too, are read, and those from k on ignored.  d_a_scales [m], d_b_scales [n], d_bias [n] (may be NULL) fp32.
 *   d_out [m][n] of out_dtype, out_stride >= n.  1 <= k <= IVFPQ_MAX_Q8_K. */
int ivfpq_q8_matmul(const int8_t* d_a, int64_t a_stride, const float* d_a_scales, int64_t m, const int8_t* d_b,
                    int64_t b_stride, const float* d_b_scales, int64_t n, int32_t k, const float* d_bias, void* d_out,
                    int32_t out_dtype, int64_t out_stride, void* hip_stream);

/* Search results as a distribution over tokens: neighbour j weighs exp(-dist_j / temperature), the weights of a query sum
 * to one, and neighbours with the same token add up.  d_ids [nq][k] i64 and d_dists [nq][k] fp32 as ivfpq_search returns
 * them; d_id_tokens [n_ids] int32: the token of every id.  A neighbour whose id is outside [0, n_ids), whose distance is not
 * finite or whose token is negative is left out.  d_tokens [nq][k] int32: the distinct tokens in the order of their first
 * neighbour, d_logprobs [nq][k] fp32 their log-probabilities; unused places hold -1 and -inf.  1 <= k <= IVFPQ_MAX_LISTED, 1e-30 <= temperature <= 1e30. */
int ivfpq_neighbour_tokens(const int64_t* d_ids, const float* d_dists, int64_t nq, int32_t k, const int32_t* d_id_tokens,
                           int64_t n_ids, float temperature, int32_t* d_tokens, float* d_logprobs, void* hip_stream);

/* Log-probability of one given token a row, entropy of the row's distribution and its `top` most likely tokens.
 *   d_logits [n][vocab]                     d_targets [n] int32, may be NULL
 *   d_logprobs [n]: of d_targets, 0 for a target outside [0, vocab); NULL if and only if d_targets is
 *   d_entropy [n] (nats), d_norms [n][2]: may be NULL
 *   d_top_tokens, d_top_logprobs [n][top]: descending, ties to the lower token; tokens whose log-probability is -inf (p = 0, or
 *   log p below every fp32 number) are not listed, and unused places hold -1 and -inf (-1 and NaN in a row of NaN statistics, whose
 *   tokens are of no meaning).  The order of the model's own distribution is that of the logits.  0 <= top <= IVFPQ_MAX_TOP.
 * n_neighbours > 0 mixes the rows' distributions with listed ones (ivfpq_neighbour_tokens): (1 - weight) p + weight q,
 * 0 < weight < 1, q given by d_neighbour_tokens and d_neighbour_logprobs [n][n_neighbours]; the used tokens of a row are
 * distinct.  Log-probabilities, entropy and alternatives are then the mixture's (norms stay the model's).  A row without
 * a used neighbour is the model's alone, a row whose logits are all -inf the neighbours' alone.
 * 0 <= n_neighbours <= IVFPQ_MAX_LISTED; where top > 0 and n_neighbours > 0, top + n_neighbours <= IVFPQ_MAX_MIXED.
 * d_workspace: >= ivfpq_token_logprobs_workspace_bytes(...) (may be 0), 256-byte aligned. */
size_t ivfpq_token_logprobs_workspace_bytes(int64_t n, int32_t vocab, int32_t top, int32_t n_neighbours);
int ivfpq_token_logprobs(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                         const int32_t* d_targets, float temperature, int32_t top, const int32_t* d_neighbour_tokens,
                         const float* d_neighbour_logprobs, int32_t n_neighbours, float weight, float* d_logprobs,
                         float* d_entropy, float* d_norms, int32_t* d_top_tokens, float* d_top_logprobs, void* d_workspace,
                         size_t workspace_bytes, void* hip_stream);

/* Gradient with respect to the logits of sum_i g_i logprob_i + h_i entropy_i (the model's own distribution, no
 * mixture), g = d_grad_logprobs [n], h = d_grad_entropy [n]; either may be NULL (zeros), not both:
 *   grad[v] = (g (v == target) - g p_v - h p_v (log p_v + entropy)) / T,  g of a target outside [0, vocab) counted as 0.
 * d_norms, d_entropy: of a forward call without neighbours (a mixture's entropy is another) on the same logits and temperature.
 * d_entropy may be NULL without d_grad_entropy, d_targets without d_grad_logprobs.  d_grad [n][vocab] of the logits' dtype. */
int ivfpq_token_logprobs_backward(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                                  const int32_t* d_targets, float temperature, const float* d_norms, const float* d_entropy,
                                  const float* d_grad_logprobs, const float* d_grad_entropy, void* d_grad,
                                  int64_t grad_stride, void* hip_stream);

/* Divergence of a student from a teacher of whom only a few tokens a row are known: with P the softmax of the listed
 * teacher_logits / T (log-probabilities serve as well) and p the student's distribution over the whole vocabulary,
 *   loss = T^2 sum_j P_j (log P_j - log p_token(j)).
 * d_teacher_tokens [n][k] int32, d_teacher_logits [n][k] fp32; entries outside [0, vocab) or at -inf are unused, entries of
 * the same token add up.  d_loss [n]: 0 without a used entry, +inf where the student gives one of them p = 0.
 * d_norms [n][2].  1 <= k <= IVFPQ_MAX_LISTED.  d_workspace: >= ivfpq_distill_topk_workspace_bytes(n, vocab), 256-byte aligned. */
size_t ivfpq_distill_topk_workspace_bytes(int64_t n, int32_t vocab);
int ivfpq_distill_topk(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                       const int32_t* d_teacher_tokens, const float* d_teacher_logits, int32_t k, float temperature,
                       float* d_loss, float* d_norms, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Gradient of sum_i w_i loss_i with respect to the logits: grad[v] = T w (p_v - P_v), 0 in rows without a used entry.
 * d_norms of the forward call; w = d_row_grads [n], NULL for ones.  d_grad [n][vocab] of the logits' dtype. */
int ivfpq_distill_topk_backward(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                                const float* d_norms, const int32_t* d_teacher_tokens, const float* d_teacher_logits,
                                int32_t k, float temperature, const float* d_row_grads, void* d_grad, int64_t grad_stride,
                                void* hip_stream);

/* Both in one call, for training steps whose row weights are known beforehand.  Workspace as ivfpq_distill_topk. */
int ivfpq_distill_topk_step(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                            const int32_t* d_teacher_tokens, const float* d_teacher_logits, int32_t k, float temperature,
                            const float* d_row_grads, float* d_loss, void* d_grad, int64_t grad_stride, void* d_workspace,
                            size_t workspace_bytes, void* hip_stream);

/* ---- drafted tokens: from the neighbours' texts, through a paged cache, to the model's verdict ----
 *
 * The text behind a stored state goes on in some way; a neighbour's continuation is a draft of what the model will say.  One pass of the
 * model then takes n sequences of m rows: row 0 the last token that was kept, the others drafts, each the successor of its parent row.
 * ivfpq_neighbour_drafts makes these trees, ivfpq_cache_append and ivfpq_draft_attention take the rows through a layer,
 * ivfpq_verify_drafts decides by the model's logits which rows are kept, and ivfpq_cache_keep closes the gaps between them in the caches.
 *
 *  - d_parents [n][m] int32: the row that a row follows, which comes before it; any value outside [0, row) marks a row that follows the
 *    cache.  NULL: a chain, every row follows the one before it (row 0 the cache).  Trees have up to IVFPQ_MAX_DRAFT rows, chains
 *    up to 2^20 where not stated otherwise (a prompt, or a piece of one).
 *  - d_counts [n] int32: a sequence's used rows are the first of them (values outside [0, m] count as the nearest); NULL: all m.  Unused rows
 *    change nothing in a cache, and nothing in them is read; what outputs hold for them is stated with each call.
 *  - The cache of one layer: d_k_cache [n_pages][kv_heads][page][d] and d_v_cache [n_pages][kv_heads][page / 8][d][8], fp16 or bf16, 16-byte
 *    aligned; values of 8 places lie side by side, so that a product over places reads 16 bytes of each component.  page: a power of two
 *    from 16 to 256; d: a multiple of 8, 8 <= d <= 256.
 *  - d_pages [n][max_pages] int32: place p of sequence s is place p % page of page d_pages[s][p / page].  d_lens [n] int32: places that
 *    the sequence has in the cache before the pass (negative values count as 0); row i is at place lens + i.  A place beyond max_pages pages, or in a
 *    page outside [0, n_pages), is not there: nothing is written to it and nothing read.  max_pages * page < 2^31 - 2^21.
 *  - The pages that hold a pass's rows belong to one sequence only, and stand once in its list.  Outputs overlap no inputs.
 *  - Limits: n <= 2^20, n * m <= 2^24, kv_heads <= 4096, heads <= 65536. */
enum {
    IVFPQ_MAX_DRAFT = 64,       /* rows of a tree */
    IVFPQ_MAX_DRAFT_DEPTH = 15, /* tokens of a continuation */
    IVFPQ_MAX_HEAD = 256        /* components of a head */
};

/* Search results as trees of drafted tokens.  Neighbour j continues with the tokens d_text[id], d_text[id + 1], ... (d_text [n_ids] int32: the
 * token that followed each stored state, states in the order of their text), up to `depth` of them, to the end of d_text or to a negative
 * token (the end of a document).  It weighs w_j = exp((d_min - d_j) / temperature), rounded to a multiple of 2^-32, d_min the smallest distance
 * of those left in: a neighbour is left out where ivfpq_neighbour_tokens leaves it out.  A node of the tree is a beginning that
 * continuations share and weighs the sum of theirs.  A query's tree is row 0 = d_last (the token that the query's state comes before), then the
 * m - 1 heaviest nodes in descending order; of equal ones the shallower comes first, then the one whose first neighbour does.
 *   d_tokens, d_parents, d_depths [nq][m] int32, d_logprobs [nq][m] fp32: a row's token, parent (-1: row 0), tokens since row 0, and the
 *   logarithm of its share of the neighbours' weight (row 0: 0); rows behind the last node hold -1, -1, 0 and -inf.  d_counts [nq] int32: rows
 *   of each tree, with row 0.
 * 1 <= k <= IVFPQ_MAX_LISTED, 1 <= depth <= IVFPQ_MAX_DRAFT_DEPTH, 1 <= m <= IVFPQ_MAX_DRAFT, 1e-30 <= temperature <= 1e30. */
int ivfpq_neighbour_drafts(const int64_t* d_ids, const float* d_dists, int64_t nq, int32_t k, const int32_t* d_text, int64_t n_ids,
                           const int32_t* d_last, double temperature, int32_t depth, int32_t m, int32_t* d_tokens,
                           int32_t* d_parents, int32_t* d_depths, float* d_logprobs, int32_t* d_counts, void* hip_stream);

/* A layer's keys and values to their places in its cache, with the rotation of their positions; queries rotated alike.
 *   d_k, d_v [n * m][kv_heads][d], d_q [n * m][heads][d] (may be NULL, then heads = 0 and d_q_out NULL) of `dtype`: any for a cache of either 16-bit
 *   type if fp32, else the cache's own; k_stride, v_stride, q_stride values from one row to the next.
 *   The position of a row is lens + d_depths[s][row] (d_depths [n][m] int32; NULL: lens + row).  The first `rotated` components of a head
 *   are turned in pairs by position * d_inv_freq[i], i < rotated / 2, fp32: pairs (2i, 2i + 1) if interleaved, else (i, i + rotated / 2).  (a, b)
 *   becomes amplitude * (a cos - b sin, b cos + a sin).  Frequencies scaled for long contexts, and the amplitude that goes with some of
 *   them, are the caller's.  Angles are formed and reduced in 64 bits, the rest is fp32, rounded once to the cache's type.
 *   0 <= rotated <= d, even; d_inv_freq may be NULL with rotated = 0.
 *   d_q_out [n * m][heads][d] of the cache's type; zeros in unused rows. */
int ivfpq_cache_append(const void* d_q, int64_t q_stride, int32_t heads, const void* d_k, int64_t k_stride, const void* d_v,
                       int64_t v_stride, int32_t dtype, int64_t n, int32_t m, const int32_t* d_depths, const int32_t* d_counts,
                       const float* d_inv_freq, int32_t rotated, int32_t interleaved, float amplitude, void* d_q_out, void* d_k_cache,
                       void* d_v_cache, int32_t cache_dtype, int64_t n_pages, int32_t kv_heads, int32_t page, int32_t d,
                       const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens, void* hip_stream);

/* Attention of the rows of a pass: row r of sequence s sees the lens[s] places of the cache before the pass, its ancestors among the rows, and
 * itself, whose keys and values ivfpq_cache_append has put there:
 *   out = sum_p softmax_p(scale * q . k_p) v_p,   lse = log sum_p exp(scale * q . k_p).
 * What a row does not see has no influence on it, NaNs and infinities included.  A row that sees nothing (its places are not
 * there) is 0 with lse = -inf; unused rows likewise.
 *   d_q [n * m][heads][d] of the cache's type, 16-byte aligned, q_stride values from one row to the next, a multiple of 8; heads a multiple of kv_heads:
 *   head h reads the keys and values of h / (heads / kv_heads).  d_out [n * m][heads][d] likewise, out_stride, 8-byte aligned.  d_lse [n * m][heads]
 *   fp32, may be NULL.
 *   max_places: about how many places the longest sequence has with its rows.  It decides how the work is divided and what workspace that needs, and nothing
 *   else: whatever it is, all places of d_pages are seen, also where a captured call is replayed over longer sequences.
 *   Probabilities are fp32; they are rounded to the cache's type as factors of the values (the sum that divides them is of unrounded ones).  An infinity among the
 *   values that a row sees makes its result infinite, or NaN where the weight rounds to 0 (in fp16 under 2^-31 of the largest).
 *   n * m * heads <= 2^26; the launch is limited to 2^23 workgroups.
 * d_workspace: >= ivfpq_draft_attention_workspace_bytes(...) (may be 0), 256-byte aligned. */
size_t ivfpq_draft_attention_workspace_bytes(int64_t n, int32_t m, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_places);
int ivfpq_draft_attention(const void* d_q, int64_t q_stride, int32_t heads, int64_t n, int32_t m, const int32_t* d_parents,
                          const int32_t* d_counts, const void* d_k_cache, const void* d_v_cache, int32_t cache_dtype, int64_t n_pages,
                          int32_t kv_heads, int32_t page, int32_t d, const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens,
                          int64_t max_places, float scale, void* d_out, int64_t out_stride, float* d_lse, void* d_workspace,
                          size_t workspace_bytes, void* hip_stream);

/* Which drafted tokens the model keeps, and what it says next.  Row i of sequence s has the logits in row s * m + i of d_logits, of the token behind
 * it; p is their distribution at this temperature.  m <= IVFPQ_MAX_DRAFT, chains too.  From row 0 on:
 *  - d_draft_logits NULL (drafts that were not drawn at random): the row's token is the lowest v with p_0 + ... + p_v > u, u = d_uniforms[s][i]
 *    (d_uniforms [n][m] fp32; NULL: the most likely token, ties to the lowest).  If a used row that follows this one holds it (the first of them
 *    that does), that row is kept and the next; otherwise it is the next token.
 *  - d_draft_logits [n * (m - 1)][vocab] of the logits' type (a chain; d_uniforms and d_accept given): row s * (m - 1) + i holds the logits from
 *    whose distribution q, at the same temperature, tokens[s][i + 1] was drawn.  Row i + 1 is kept if d_accept[s][i + 1] * q_x < p_x, x its token.
 *    Otherwise the next token is drawn like above from max(p - q, 0) divided by its sum (from p if that is 0); behind
 *    the last used row from p.  A row of draft logits without a distribution counts as q = 0.
 * Either way what is said has the distribution of the model without drafts, if the random numbers are independent and uniform on [0, 1) (others count as
 * the nearest number there, NaN as 0).  Sums are of 64 bits.
 *   d_tokens [n][m] int32; d_tokens[s][0] is not looked at
 *   d_path [n][m] int32: the kept rows, 0 first; then -1.  d_kept [n] int32: how many; 0 for a sequence without used rows.
 *   d_next [n] int32: the token behind the last kept row; -1 without used rows, and where that row has no distribution or NaN statistics
 *   d_logprobs [n][m] fp32: log p of the token behind each kept row (NaN in a row of NaN statistics); -inf in unused places.
 * 1e-6 <= temperature <= 1e6; n * m <= 2^20, vocab <= 2^30, and n * m times the 2048s in vocab + 7 <= 2^24.
 * d_workspace: >= ivfpq_verify_drafts_workspace_bytes(...), 256-byte aligned; with_drafts: d_draft_logits is given. */
size_t ivfpq_verify_drafts_workspace_bytes(int64_t n, int32_t m, int32_t vocab, int32_t with_drafts);
int ivfpq_verify_drafts(const void* d_logits, int32_t dtype, int64_t n, int32_t m, int32_t vocab, int64_t row_stride,
                        const int32_t* d_tokens, const int32_t* d_parents, const int32_t* d_counts, const float* d_uniforms,
                        double temperature, const void* d_draft_logits, int64_t draft_stride, const float* d_accept, int32_t* d_path,
                        int32_t* d_kept, int32_t* d_next, float* d_logprobs, void* d_workspace, size_t workspace_bytes,
                        void* hip_stream);

/* The kept rows move up behind each other: place lens + d_path[s][i] goes to lens + i, i < d_kept[s], in every layer.
 * d_path [n][m] int32, ascending, d_kept [n] int32 as ivfpq_verify_drafts gives them: entries outside [i, m) move nothing.
 * d_k_cache, d_v_cache: layers caches behind each other (all with the same pages); layers <= 4096, layers * kv_heads * d <= 2^31.  The sequence's length is the caller's to raise by d_kept. */
int ivfpq_cache_keep(void* d_k_cache, void* d_v_cache, int32_t cache_dtype, int32_t layers, int64_t n_pages, int32_t kv_heads, int32_t page,
                     int32_t d, const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens, int64_t n, int32_t m,
                     const int32_t* d_path, const int32_t* d_kept, void* hip_stream);

/* ---- measurement aid ---- */

/* When enabled, search calls record HIP events around their stages on the stream they run on (the events
 * and their bookkeeping live in the handle: while enabled, search calls on one index must not overlap).
 * After the stream has been synchronised, ivfpq_stage_times_ms reports the last call's
 * milliseconds, summed over query tiles: ms[0] = probe selection (step 1: ranking GEMM + selection),
 * ms[1] = table build + code scan (steps 2-4: the scan of the nearest probes and their bound, the grouping of the
 * other pairs by cluster, the scan of the remaining probes), ms[2] = top-k (step 5), ms[3] = whole call; and
 * parts of those stages: ms[4] = the ranking GEMM of step 1, ms[5] = the scan of the nearest probes with its
 * bound (one launch, or in large batches three: the queries' order, the scan of up to four at once, the
 * bound), ms[6] = the scan of the remaining probes (the dominant kernel, or two), ms[7] = of ms[5] the bound where it
 * is a launch of its own, else 0.  Small searches scan all probes in one launch: its
 * time is divided between ms[5] and ms[6] by the number of pairs, 1 : n_probes - 1. */
int ivfpq_set_stage_timing(ivfpq_index_t* index, int32_t enabled);
int ivfpq_stage_times_ms(ivfpq_index_t* index, float ms[8]);

/* Writes into buf (host, buf_bytes > 0, always terminated) the name, workgroup size and LDS request of the
 * kernel that scans the probes other than the nearest one (the dominant kernel of a search): what to look for in a
 * profiler's kernel list.  While stage timing is enabled and the last search used this table dtype, it is what that
 * search launched (its first query tile).  Otherwise it describes large batches on this index with the current tuning,
 * whose pairs run grouped by cluster, unless IVFPQ_TUNE_SCAN_ROUTE names another route.  Where a matrix product can list
 * the vectors to add up (an uploaded index, its usual shapes, no knob that asks for the table kernels) that names its
 * kernel and the one that adds them up; a search for which the tables cost less (few vectors looked up, or many of them
 * able to be among the results) takes the table kernels all the same, and one of little work scan_kernel. */
int ivfpq_scan_kernel_info(const ivfpq_index_t* index, int32_t lut_dtype, char* buf, size_t buf_bytes);

/* Measurement aid, not a step of the method: a plain streaming read of `bytes` bytes of device memory
 * (16-byte loads, grid-strided, n_out workgroups of 256 threads), the achievable HBM read rate that a
 * code scan (Sec. I-C, search step 4, Eq. 1) streaming every byte from HBM is priced against.  d_buf: device,
 * 16-byte aligned, bytes a multiple of 16; d_out: device, n_out words (1..65536), word b = XOR of all
 * 32-bit words workgroup b read.  Asynchronous on hip_stream; allocates nothing. */
int ivfpq_stream_read(const void* d_buf, size_t bytes, uint32_t* d_out, int32_t n_out, void* hip_stream);

const char* ivfpq_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* IVFPQ_H */
