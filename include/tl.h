/*
 * tl.h -- C ABI of the MI355X (gfx950) library for the batched hot path of
 * throttLL'eM's per-iteration GPU-frequency controller (arXiv 2408.05235).
 *
 * For many independent what-if scenarios the library runs three stages, each
 * a HIP kernel on one device:
 *   tl_project        projected batch size and KV-cache blocks per future
 *                     iteration (Sec. 4.2, Eq. 1-2), with FIFO admission of
 *                     queued requests under the KV check of Sec. 4.3.2;
 *                     optionally the feature rows of the performance model;
 *   tl_forest_predict the performance model M, a gradient-boosted tree
 *                     ensemble predicting iterations per second (Sec. 4.3.1);
 *   tl_select_freq    the throttling controller (Sec. 4.5): per scenario the
 *                     lowest frequency whose predicted per-iteration times
 *                     pass the TBT check and the E2E deadlines (Sec. 4.3.2,
 *                     checks 2 and 3, Eq. 3-4).
 * and, from the same stages, tl_select_freq_binary (the controller's binary
 * search as the paper states it, querying the model only at probed
 * frequencies) and tl_admit (the admission control of Sec. 4.3.2 for one new
 * query per scenario).  Below them stands the machine that they plan: the paged
 * cache whose blocks tl_project counts (tl_pages_*, tl_kv_append) and the
 * attention over it (tl_attend).
 *
 * Conventions shared by every entry point
 *   - Pointers are DEVICE pointers (memory of the device that is current on
 *     the calling thread) owned by the caller, unless the comment says host.
 *     The library never frees or retains caller memory.
 *   - `stream` is a hipStream_t (NULL = the legacy default stream).  Calls
 *     only enqueue work; none synchronizes.  Outputs are valid once the
 *     stream reaches that point.
 *   - Argument errors (sizes, NULL pointers, unsupported shapes) are detected
 *     on the host before anything is enqueued and return TL_EINVAL; nothing
 *     is written.  A failed HIP call returns TL_EDEVICE.  tl_last_error()
 *     then describes the failure (thread-local, valid until the next call).
 *   - Data-dependent anomalies never fail a call: they are reported per
 *     scenario through TL_FLAG_* bits and TL_STATUS_* values.
 *   - Results are deterministic: bit-identical across runs and launches.
 *   - A call takes up to 2^26 - 4 scenarios (memory permitting; feature rows
 *     written out and table lookups: scenarios x 256 iterations); launches of
 *     more fail with TL_EDEVICE.
 */
#ifndef TL_H
#define TL_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TL_ABI_VERSION 1

typedef enum tl_status {
    TL_OK = 0,
    TL_EINVAL = 1,          /* invalid argument; nothing was enqueued          */
    TL_ENOMEM = 2,          /* device allocation failed                        */
    TL_EDEVICE = 3,         /* a HIP runtime call or kernel launch failed      */
    TL_EUNSUPPORTED = 4     /* valid but beyond the library's limits          */
} tl_status;

/* Limits of the library. */
#define TL_MAX_HORIZON 8192         /* H: future iterations per scenario      */
#define TL_MAX_BLOCK_TOKENS 65536   /* N: tokens per KV block                 */
#define TL_MAX_FREQS 4096           /* F: candidate frequencies               */
#define TL_MAX_FEATURES 4           /* model inputs (Sec. 4.3.1 lists four)   */
#define TL_MAX_DEPTH 14             /* tree depth                             */

/* Per-scenario flags written by tl_project (bitwise OR). */
#define TL_FLAG_BAD_REQUEST 1u  /* some scoreboard entries were malformed and ignored:
                                   prompt < 0, generated < 0, remaining < 1,
                                   arrival < -1, or prompt + generated > 2^30 */
#define TL_FLAG_LOST        2u  /* an in-flight request is marked lost (Sec. 4.3.2)   */
#define TL_FLAG_OVERCOMMIT  4u  /* the in-flight batch alone exceeds the KV capacity
                                   at some iteration, or exceeds the batch cap now    */
#define TL_FLAG_OVERFLOW    8u  /* scenario not projected: its request range is
                                   invalid, or sum over valid entries of
                                   ceil((prompt+generated+H)/N) > 2^31-1, so curves
                                   could overflow; outputs are zero / no deadline  */
#define TL_FLAG_UNSORTED   16u  /* queued entries are not in non-decreasing arrival
                                   order; the queue is still served in array order */
#define TL_FLAG_BAD_CANDIDATE 32u /* tl_admit only: the new query is malformed
                                   (prompt < 0 or > 2^30, length < 1) and was left
                                   out of the projection */

/* Per-scenario status written by tl_select_freq. */
#define TL_STATUS_OK         0u  /* freq_idx is the lowest feasible index           */
#define TL_STATUS_INFEASIBLE 1u  /* no frequency passes; freq_idx = F-1            */
#define TL_STATUS_LOST       2u  /* a lost request forces the maximum; freq_idx = F-1 */
#define TL_STATUS_INVALID    3u  /* scenario flagged TL_FLAG_OVERFLOW; freq_idx = F-1 */

/* Per-scenario decision written by tl_admit (Sec. 4.3.2). */
#define TL_ADMIT_OK             0u  /* checks 1-3 pass: schedule the query            */
#define TL_ADMIT_LOST           1u  /* only its own deadline fails: schedule it and
                                       mark it lost                                   */
#define TL_ADMIT_QUEUE_CAPACITY 2u  /* check 1: a projected KV value exceeds the
                                       capacity, or the batch running now exceeds
                                       the batch cap -> queue                         */
#define TL_ADMIT_QUEUE_TBT      3u  /* check 2: mean TBT at the maximum frequency
                                       exceeds the SLO -> queue                       */
#define TL_ADMIT_QUEUE_E2E      4u  /* check 3: a scheduled request would miss its
                                       deadline (Eq. 4) -> queue                      */
#define TL_ADMIT_INVALID        5u  /* malformed query or scenario not projected     */

/* Per-iteration time that stands for "no progress" (IPS <= 0, NaN, or
 * 1e9/IPS >= 2^40 ns). */
#define TL_LAT_SATURATED_NS (1ull << 40)
#define TL_NO_DEADLINE UINT64_MAX

int32_t tl_abi_version(void);        /* returns TL_ABI_VERSION */
const char* tl_last_error(void);     /* message for the last non-OK status on this thread */

/* ------------------------------------------------------------------------
 * The performance model M (Sec. 4.3.1): a gradient-boosted decision-tree
 * ensemble over the inputs the paper names (engine size, batch size, KV-cache
 * usage, GPU frequency) that predicts iterations per second.
 *
 * Trees are complete, of depth `depth`, in heap order: internal node k
 * (0 <= k < 2^depth - 1) compares x[feature[k]] < threshold[k] in fp32 and
 * continues at 2k+1 when true, 2k+2 otherwise (a NaN input goes to 2k+2);
 * after `depth` comparisons the node index minus (2^depth - 1) selects one of
 * the 2^depth leaves.  A shallower tree is expressed by padding with
 * threshold +inf (always 2k+1).  The prediction of a row is base_score plus
 * the selected leaf of every tree as an fp32 running sum in tree order
 * (acc = base_score, then acc += leaf_t for t = 0 .. n_trees-1, each add
 * rounded to nearest even): the paper does not state the sum's precision,
 * and this is how an ensemble that keeps its predictions in fp32 adds them.
 *
 * feature   host, uint8 [n_trees][2^depth - 1], each < n_features
 * threshold host, fp32  [n_trees][2^depth - 1]
 * leaf      host, fp32  [n_trees][2^depth]
 * The arrays are copied to the current device; the handle owns that copy and
 * must be used with the same device.  n_trees >= 0 (0 gives base_score),
 * 0 <= depth <= TL_MAX_DEPTH, 1 <= n_features <= TL_MAX_FEATURES.
 * Errors: TL_EINVAL (bad sizes, NULL, feature index out of range),
 * TL_ENOMEM, TL_EDEVICE.  On error *out is set to NULL.
 * ---------------------------------------------------------------------- */
typedef struct tl_forest tl_forest;

tl_status tl_forest_create(int32_t n_trees, int32_t depth, int32_t n_features, float base_score,
                           const uint8_t* feature, const float* threshold, const float* leaf,
                           tl_forest** out);
void tl_forest_destroy(tl_forest* forest);   /* NULL is ignored; synchronizes the device */

/* ------------------------------------------------------------------------
 * Scoreboard lengths under generation-length errors (Sec. 4.6): the
 * remaining-token counts tl_project takes, from the predictor's total
 * generation lengths.  Per request i of scenario s (CSR req_offset as in
 * tl_project):
 *   len = ceil(pred_len[i] * scale_num[s] / scale_den[s])   (scale_den 0: pred_len)
 *   len = min(len, max_tokens[s]);  if generated[i] >= len: len = max_tokens[s]
 *                                                   (both only when max_tokens[s] >= 1)
 *   remaining_out[i] = max(len - generated[i], 1)
 * Entries with generated < 0 or pred_len < 1 get 0, which tl_project ignores
 * as malformed.  Scenarios whose request range is invalid are not written.
 * remaining_out may alias neither input.
 * ---------------------------------------------------------------------- */
tl_status tl_adjust_lengths(int64_t n_scenarios, int64_t n_requests, const int64_t* req_offset,
                            const int32_t* generated, const int32_t* pred_len, const uint32_t* scale_num,
                            const uint32_t* scale_den, const int32_t* max_tokens, int32_t* remaining_out,
                            void* stream);

/* ------------------------------------------------------------------------
 * Stage 1 -- KV usage and batch-size projection (Sec. 4.2, Eq. 1-2).
 *
 * Scenario s owns requests req_offset[s] .. req_offset[s+1]-1 (a scoreboard,
 * Table 1).  Iterations are relative: j = 0 is the current iteration k.
 * Request i has prompt length |q_i| = prompt_len[i], has generated
 * generated[i] tokens and is projected to need remaining[i] more iterations.
 *   arrival_iter[i] == -1 : in the batch now (scheduled g_i iterations ago);
 *                           it occupies iterations [0, remaining[i]).
 *   arrival_iter[i] >= 0  : queued; it becomes eligible at that iteration.
 * Queued entries form one FIFO in array order.  At iteration j, after the
 * requests ending at j leave, the head joins (s_a = j, its lifetime is
 * [j, j + remaining)) iff it has arrived, the batch at j is below
 * batch_cap[s], and appending it keeps every projected KV value from j to
 * H-1 at or below kv_capacity[s] (Sec. 4.3.2 check 1); several may join at the
 * same j; a head that cannot join blocks the queue.
 *
 * Outputs ([s][j] row-major, j < H):
 *   batch[s][j]       number of requests in the batch at iteration j
 *   kv[s][j]          KV blocks in use: sum of ceil((prompt + generated +
 *                     (j - start)) / N) over those requests (Eq. 1-2)
 *   deadline_at[s][j] minimum deadline_ns over non-lost requests whose last
 *                     iteration in the batch is j (finishing inside the
 *                     horizon), TL_NO_DEADLINE if none (Eq. 4 checkpoints)
 *   n_iters[s]        number of projected iterations: min(H, last finish)
 *   flags[s]          TL_FLAG_* bits
 * Optional feature rows (rows != NULL), [s][f][j][n_features] fp32:
 *   (freqs_mhz[f], kv[s][j], batch[s][j] [, engine_size[s]])
 * the query vector of Sec. 4.3.2 check 2 for every candidate frequency.
 * freqs_mhz must be ascending; index F-1 is the maximum frequency.
 *
 * Scoreboards with long FIFO loops (no batch_cap and on average 1024 or more
 * requests per scenario) are projected heaviest first (results do not depend
 * on the order).  The order takes 4 bytes per scenario of device scratch
 * that the library owns, one per device: allocated on the first such call,
 * kept, and replaced only when more scenarios come (as the forest's, see
 * tl_forest_predict_grid; without ever waiting on the host).  If that allocation
 * fails the scenarios run in their own order (same results), as they do
 * while the stream is being captured into a graph.  Calls share it: a call
 * on another stream than the previous one first waits (on the device) for
 * the previous projection.
 * ---------------------------------------------------------------------- */
typedef struct tl_project_args {
    uint32_t struct_size;          /* sizeof(tl_project_args) */
    int32_t horizon;               /* H, 1 .. TL_MAX_HORIZON */
    int64_t n_scenarios;           /* S >= 0 */
    int64_t n_requests;            /* total entries; req_offset[S] must equal it */
    int32_t block_tokens;          /* N, 1 .. TL_MAX_BLOCK_TOKENS */
    int32_t n_freqs;               /* F (rows only), 1 .. TL_MAX_FREQS */
    int32_t n_features;            /* 3 or 4 (rows only) */
    int32_t reserved;
    const int64_t* req_offset;     /* [S+1] */
    const int32_t* prompt_len;     /* [n_requests] */
    const int32_t* generated;      /* [n_requests] */
    const int32_t* remaining;      /* [n_requests] */
    const int32_t* arrival_iter;   /* [n_requests] */
    const uint64_t* deadline_ns;   /* [n_requests], t_dead - t_cur in ns; NULL = none */
    const uint8_t* lost;           /* [n_requests], nonzero = lost; NULL = none */
    const int32_t* kv_capacity;    /* [S] blocks */
    const int32_t* batch_cap;      /* [S]; NULL = unlimited */
    int32_t* batch;                /* out [S][H] */
    int32_t* kv;                   /* out [S][H] */
    uint64_t* deadline_at;         /* out [S][H] */
    int32_t* n_iters;              /* out [S] */
    uint32_t* flags;               /* out [S] */
    const float* freqs_mhz;        /* [F] (rows only) */
    const float* engine_size;      /* [S] (rows with n_features == 4) */
    float* rows;                   /* out [S][F][H][n_features]; NULL = no rows */
} tl_project_args;

tl_status tl_project(const tl_project_args* args, void* stream);

/* ------------------------------------------------------------------------
 * Stage 2 -- the model M on arbitrary feature rows (Sec. 4.3.1).
 * rows [n_rows][n_features of the forest] fp32 row-major; out [n_rows] fp32.
 * Calls with few rows (here, on the grid and at one frequency per scenario)
 * of forests with many trees are cut along the trees as well and take up to 64
 * MiB of the forest handle's device scratch (tl_forest_predict_grid says how it
 * is kept); without it, or under stream capture, they give the same results in
 * more time.
 * ---------------------------------------------------------------------- */
tl_status tl_forest_predict(const tl_forest* forest, const float* rows, int64_t n_rows,
                            float* out, void* stream);

/* ------------------------------------------------------------------------
 * Stage 2 on the projection grid, fused with the row expansion: the same
 * values tl_forest_predict gives for the rows tl_project would write, without
 * materializing them (Sec. 4.3.2 check 2 and Sec. 4.5 query M for every
 * projected iteration at every candidate frequency).
 *   out[s][f][j] = M(freqs_mhz[f], kv[s][j], batch[s][j] [, engine_size[s]])
 * freqs_mhz [F]; kv, batch [S][H] int32 as written by tl_project (converted
 * to fp32); engine_size [S], required when the forest has 4 features and
 * ignored otherwise; out [S][F][H] fp32.  The forest must have 3 or 4
 * features in the order (frequency, KV, batch[, engine size]).
 * 1 <= F <= TL_MAX_FREQS, 1 <= H <= TL_MAX_HORIZON.
 * Work on grids of more than two workgroups per CU is ordered by an estimate
 * of its cost (results do not depend on the order).  The ordering needs 16
 * bytes per (scenario, 64-iteration chunk) plus a radix sort's temporary
 * storage of device scratch, which the forest handle owns: up to four arrays,
 * allocated when a call first needs one, kept, and replaced only when a larger
 * call comes, so repeated calls of one size allocate nothing.  Arrays are
 * powers of two in size, and a replaced one is freed with the handle, so
 * that a larger call does not wait on the host either (only where no memory is
 * left does it free the replaced arrays first, which waits).  If that
 * allocation fails, or the stream is being captured into a graph, the call
 * runs without the ordering (same results; tl_forest_predict_grid_noalloc
 * keeps it under capture).  A call takes the array its stream used last, or an
 * idle one; when four other streams' calls still use all of them it first
 * waits (on the device) for the previous call's work.  (On hipStreamPerThread
 * every thread has a stream of its own.)  The forest's device
 * must be the current device.
 * ---------------------------------------------------------------------- */
tl_status tl_forest_predict_grid(const tl_forest* forest, int64_t n_scenarios, int32_t n_freqs,
                                 int32_t horizon, const float* freqs_mhz, const int32_t* kv,
                                 const int32_t* batch, const float* engine_size, float* out,
                                 void* stream);

/* ------------------------------------------------------------------------
 * tl_forest_predict_grid for callers that cannot allocate device memory
 * (code under stream capture, tight serving loops, hosts that forbid
 * allocation): same arguments, same results, no allocation of any kind.
 * The work order's scratch is a fixed 32 MiB array of the library on each
 * device (taken when the library is loaded): 16 bytes per (scenario,
 * 64-iteration chunk) pair plus the sort's temporary storage must fit, as
 * they do for 16384 scenarios x 2048 iterations (524,288 pairs) but not for
 * 65536 x 2048.  A grid whose order needs more returns TL_EUNSUPPORTED and
 * enqueues nothing.  Every call on one device shares that array: calls that
 * overlap on one device (concurrent streams, other threads) race and must
 * be serialized by the caller; tl_forest_predict_grid does not use it.
 * ---------------------------------------------------------------------- */
tl_status tl_forest_predict_grid_noalloc(const tl_forest* forest, int64_t n_scenarios, int32_t n_freqs,
                                         int32_t horizon, const float* freqs_mhz, const int32_t* kv,
                                         const int32_t* batch, const float* engine_size, float* out,
                                         void* stream);

/* ------------------------------------------------------------------------
 * Stage 2 through a table: the model compiled to its discrete input lattice.
 * The controller queries M only at a fixed list of frequencies, a few engine
 * sizes, integer batch sizes and integer KV blocks (Sec. 4.3.1 notes that
 * all inputs are bounded), so M can be evaluated once at every lattice point
 * and prediction becomes a table lookup:
 *   tl_lattice_create evaluates M (with tl_forest_predict_grid's kernels, so
 *   every value is the fp32 tree-order sum a walk gives) at every
 *   (engine size, batch 0..batch_max, frequency, KV 0..kv_max); the table
 *   takes n_engines x (batch_max + 1) x n_freqs x 4096 x ceil((kv_max + 1) /
 *   4096) x 4 bytes (tl_lattice_bytes), at most 256 GiB.
 *   tl_lattice_predict_grid gives out[s][f][j] exactly as
 *   tl_forest_predict_grid with the lattice's frequencies: lattice points are
 *   read from the table, other rows (KV or batch outside [0, max], an engine
 *   size not in the list) are walked.
 * freqs_mhz: device [n_freqs], copied.  engine_values: host
 * [n_engines <= 16], required for 4-feature forests (ignored otherwise).
 * The build is enqueued on `stream`, which the call synchronizes once (to
 * keep a host copy of the frequency list); the forest must outlive the
 * lattice.
 * Errors: TL_EINVAL, TL_EUNSUPPORTED (table too large), TL_ENOMEM,
 * TL_EDEVICE.
 * ---------------------------------------------------------------------- */
typedef struct tl_lattice tl_lattice;

tl_status tl_lattice_create(const tl_forest* forest, int32_t n_freqs, const float* freqs_mhz, int32_t n_engines,
                            const float* engine_values, int32_t kv_max, int32_t batch_max, void* stream,
                            tl_lattice** out);
void tl_lattice_destroy(tl_lattice* lattice);   /* NULL is ignored; synchronizes the device */
uint64_t tl_lattice_bytes(const tl_lattice* lattice);
tl_status tl_lattice_predict_grid(const tl_lattice* lattice, int64_t n_scenarios, int32_t horizon,
                                  const int32_t* kv, const int32_t* batch, const float* engine_size, float* out,
                                  void* stream);

/* ------------------------------------------------------------------------
 * Stage 3 -- frequency selection (Sec. 4.5 with Sec. 4.3.2 checks 2-3).
 *
 * ips [S][F][H] fp32: predicted iterations/s of scenario s at frequency f in
 * iteration j.  With n = clamp(n_iters[s], 0, H) and per-iteration times
 * lat = ceil(1e9 / ips) ns (one IEEE fp64 division; TL_LAT_SATURATED_NS for
 * ips <= 0, NaN or 1e9/ips >= 2^40), and T_R[l] = lat[0] + ... + lat[l-1]
 * (Eq. 3), frequency f is feasible iff n == 0, or
 *   T_R[n] <= tbt_slo_ns[s] * n            (mean TBT, check 2), and
 *   T_R[j+1] < deadline_at[s][j] for every j < n with a deadline (Eq. 4).
 * freq_idx[s] = lowest feasible f (status OK), else F-1 (INFEASIBLE).  If
 * proj_flags[s] has TL_FLAG_OVERFLOW: F-1, INVALID; else if it has
 * TL_FLAG_LOST: F-1, LOST (the search is bypassed).  proj_flags may be NULL.
 * ---------------------------------------------------------------------- */
tl_status tl_select_freq(const float* ips, int64_t n_scenarios, int32_t n_freqs, int32_t horizon,
                         const uint64_t* deadline_at, const int32_t* n_iters,
                         const uint64_t* tbt_slo_ns, const uint32_t* proj_flags,
                         int32_t* freq_idx, uint32_t* status, void* stream);

/* ------------------------------------------------------------------------
 * The paper's throttling controller as it states it (Sec. 4.5): a binary
 * search over the candidate frequencies that queries the model only at the
 * frequency each scenario probes.  Per scenario, with lo = 0, hi = F-1:
 * while lo < hi, mid = lo + (hi - lo) / 2, M on every projected iteration at
 * freqs_mhz[mid], feasible as in tl_select_freq -> hi = mid, else lo =
 * mid + 1; finally lo is checked: feasible -> freq_idx = lo (OK), else F-1
 * (INFEASIBLE).  Flags as in tl_select_freq (OVERFLOW -> INVALID, LOST ->
 * F-1 without a search).  It equals tl_select_freq whenever feasibility is
 * monotone in the frequency, and evaluates M on at most ceil(log2 F) + 1
 * rows per (scenario, iteration) instead of F: the check of lo evaluates
 * nothing new when hi has moved below F-1, since hi only moves to a probe
 * found feasible and then lo == hi.
 * kv, batch, deadline_at, n_iters, proj_flags: as written by tl_project;
 * freqs_mhz [F] ascending; engine_size [S] for 4-feature forests.
 * Work arrays of the caller: ips_work [S][H] fp32 (left holding, per
 * scenario, M at the last frequency it evaluated; rows of scenarios flagged
 * lost or overflow are not written) and search_work [3][S] int32.
 * On grids that give every CU at least two workgroups of the model's kernel
 * (16 wavefronts of 64 lanes x 16, else 8, consecutive iterations of one
 * scenario), the wavefronts' work is ordered by an estimate of its cost,
 * computed once per call, and the check of lo runs only the wavefronts of
 * scenarios that need an evaluation, compacted (results depend on neither).
 * Scratch: 20 bytes per wavefront plus a radix sort's temporary storage, in
 * the forest's device scratch, as for tl_forest_predict_grid (the larger of
 * the two needs is kept; neither ordering nor compaction under stream
 * capture or without the scratch).  With few rows (S x H) and many trees the
 * model's evaluations take up to 64 MiB of it instead (tl_forest_predict).
 * Nothing else is allocated.
 * lattice (nullable): a table of the same forest and frequency count
 * (tl_lattice_create; TL_EINVAL otherwise); M at the probes is then read
 * from it, at the lattice's own frequencies (the same values when it was
 * built for freqs_mhz, which is the caller's to ensure: the list itself is
 * not compared).
 * ---------------------------------------------------------------------- */
tl_status tl_select_freq_binary(const tl_forest* forest, int64_t n_scenarios, int32_t n_freqs, int32_t horizon,
                                const float* freqs_mhz, const int32_t* kv, const int32_t* batch,
                                const float* engine_size, const uint64_t* deadline_at, const int32_t* n_iters,
                                const uint64_t* tbt_slo_ns, const uint32_t* proj_flags, float* ips_work,
                                int32_t* search_work, int32_t* freq_idx, uint32_t* status,
                                const tl_lattice* lattice, void* stream);

/* ------------------------------------------------------------------------
 * Admission control (Sec. 4.3.2) for one new query per scenario, as a batch
 * of what-ifs: the projection of tl_project on the scenario's scoreboard with
 * the query appended as a request that starts now (prompt cand_prompt[s],
 * nothing generated, active for the cand_len[s] iterations [0, L); queued and
 * arriving entries keep their FIFO admission behind it), the model at
 * max_freq_mhz on every projected iteration, and the paper's three checks in
 * order (the first failure decides):
 *   1. some projected KV value exceeds kv_capacity, or the batch running now
 *      exceeds batch_cap                         -> TL_ADMIT_QUEUE_CAPACITY
 *   2. with n = n_iters[s] and T_R as in tl_select_freq (Eq. 3),
 *      T_R[n] > tbt_slo_ns[s] * n (mean TBT)     -> TL_ADMIT_QUEUE_TBT
 *   3. T_R[e] < deadline fails for a scheduled, non-lost request ending at
 *      e <= H (Eq. 4)                            -> TL_ADMIT_QUEUE_E2E
 *      else, when L <= H and cand_deadline_ns[s] is set, T_R[L] <
 *      cand_deadline_ns[s] fails                 -> TL_ADMIT_LOST
 *   otherwise                                    -> TL_ADMIT_OK
 * A malformed query (flag TL_FLAG_BAD_CANDIDATE) or a scenario flagged
 * TL_FLAG_OVERFLOW gives TL_ADMIT_INVALID.
 *
 * `proj` describes the scoreboards and receives the projection with the query
 * (batch, kv, deadline_at without the query's deadline, n_iters, flags);
 * its rows, n_freqs, freqs_mhz and n_features are ignored.  engine_size [S]
 * is read for 4-feature forests.  ips [S][H] receives M at max_freq_mhz (rows
 * of scenarios flagged TL_FLAG_OVERFLOW hold M on the zero curves).  All
 * arrays are device arrays of the caller; the only scratch is the
 * projection's scenario order, as for tl_project, and the model kernel's
 * work order or, with few rows, its leaf values, as for
 * tl_select_freq_binary.
 * Errors as for tl_project, plus a NULL forest, ips, decision, tbt_slo_ns,
 * cand_prompt or cand_len, or a forest without 3 or 4 features: TL_EINVAL.
 * ---------------------------------------------------------------------- */
typedef struct tl_admit_args {
    uint32_t struct_size;              /* sizeof(tl_admit_args) */
    uint32_t reserved;
    tl_project_args proj;              /* scoreboards; projection outputs */
    const tl_forest* forest;
    float max_freq_mhz;                /* the maximum available frequency */
    const float* engine_size;          /* [S], 4-feature forests */
    const uint64_t* tbt_slo_ns;        /* [S] */
    const int32_t* cand_prompt;        /* [S] prompt tokens of the new query */
    const int32_t* cand_len;           /* [S] its predicted length, >= 1 */
    const uint64_t* cand_deadline_ns;  /* [S] t_dead - t_cur; NULL or TL_NO_DEADLINE = none */
    float* ips;                        /* out [S][H] */
    uint32_t* decision;                /* out [S], TL_ADMIT_* */
    const tl_lattice* lattice;         /* nullable: a table of the same forest; used
                                          when max_freq_mhz is one of its frequencies */
} tl_admit_args;

tl_status tl_admit(const tl_admit_args* args, void* stream);

/* ------------------------------------------------------------------------
 * The paged cache whose blocks tl_project counts (Sec. 4.2), and the
 * attention that reads it: the part of an engine's iteration whose time goes
 * with the batch and its KV blocks, which M is trained on (Sec. 4.3.1).
 *
 * A cache layer is a pool of n_pages pages of page_tokens tokens (the
 * projection's blocks of N tokens).  Token t of sequence b is row t % N of
 * page page_table[b][t / N]; length[b] tokens of b are in the cache.  A table
 * entry outside [0, n_pages) has no page: such tokens are neither written nor
 * seen.  Tokens past table_width * N do not exist, and a negative length is 0.
 * Keys and values have the same layout: element d of token row r of head g of
 * page p is at p * page_stride + g * head_stride + r * token_stride + d
 * (elements), so pages may be [head][token] or [token][head].  Strides are
 * multiples of 8 elements, pointers 16-byte aligned, and head_dim is a
 * multiple of 8 of at most TL_MAX_HEAD_DIM.  Offsets are 64-bit.
 *
 * New tokens come as rows of a packed array: sequence b has the rows
 * q_offset[b] .. q_offset[b+1]-1 (non-decreasing; clamped into [0, n_tokens]),
 * or row b alone when q_offset is NULL (n_tokens == n_seqs).  They are the last
 * ones of the sequence: with n rows, row i is at position length[b] - n + i
 * (length counts them already); rows of a negative position are not written
 * and see nothing.
 * ---------------------------------------------------------------------- */
#define TL_BF16 1
#define TL_F16  2
#define TL_MAX_HEAD_DIM 256

typedef struct tl_kv_view {
    uint32_t struct_size;          /* sizeof(tl_kv_view) */
    int32_t dtype;                 /* TL_BF16 or TL_F16 */
    int32_t n_kv_heads;            /* >= 1 */
    int32_t head_dim;              /* D */
    int32_t page_tokens;           /* N, 1 .. TL_MAX_BLOCK_TOKENS */
    int32_t table_width;           /* entries per table row, >= 0 */
    int64_t n_pages;               /* 0 .. 2^31-1 */
    int64_t n_seqs;                /* B >= 0 */
    int64_t page_stride;
    int64_t head_stride;
    int64_t token_stride;
    void* key_pages;               /* written by tl_kv_append only */
    void* value_pages;
    const int32_t* page_table;     /* [B][table_width] */
    const int32_t* length;         /* [B] */
} tl_kv_view;

/* A sequence whose tokens got no room has rows all the same, and a length that
 * does not count them: taken for its last tokens they would be written over
 * those that it, or a sequence that shares the page, has.  `granted` [n_seqs + 1]
 * (tl_pages_extend's; nullable) says what each got since the last append; a sequence
 * with more rows than that has no position for any of them: they are not written
 * and, where it was refused, see nothing. */

/* New keys and values to their pages: row i of key and value (strides in
 * elements between tokens and heads, multiples of 8) to its sequence's
 * position.  A page that two rows write (a shared page: fork copies those) gets
 * one of them.  Sets granted[n_seqs]. */
typedef struct tl_kv_append_args {
    uint32_t struct_size;          /* sizeof(tl_kv_append_args) */
    uint32_t reserved;
    tl_kv_view cache;
    int64_t n_tokens;              /* T >= 0 */
    const int64_t* q_offset;       /* [B+1]; NULL = one token each */
    const void* key;               /* [T][n_kv_heads][D] */
    const void* value;
    int64_t key_token_stride, key_head_stride;
    int64_t value_token_stride, value_head_stride;
    int32_t* granted;              /* [n_seqs + 1], nullable (absent: a struct_size without it) */
} tl_kv_append_args;

tl_status tl_kv_append(const tl_kv_append_args* args, void* stream);

/* Attention of the new tokens over their sequences' cached ones, the new ones
 * included (append them first).  Query head h reads KV head h / (n_heads /
 * n_kv_heads).  The token at position p sees the cached tokens t <= p, with
 * window W > 0 only those with t > p - W or t < sinks (a sliding window and a few
 * first tokens that stay visible):
 *   out = sum_t w_t v_t,  w = softmax over the visible t of scale * (q . k_t)
 *   lse = log sum_t exp(scale * (q . k_t))
 * A row that sees no token, or whose scores are all -inf, gives zeros and lse
 * -inf.  What lies in pages beyond the visible tokens, infinities and NaN
 * included, is not used.  Rows that belong to no sequence are left alone.
 *
 * Scores, the softmax's maximum and sum and the output's sums are fp32 (sum w v
 * before its division by sum w, with a largest weight of at most 1).  The
 * weights are rounded to the cache's type for the product with the values (in f16
 * scaled up, so that small ones do not vanish), the output once at the end.
 * workspace: device memory of the caller, 16-byte aligned, for the parts of
 * sequences that are split over their length and joined;
 * tl_attend_workspace_bytes(args) says how much a call can use.  With less, or
 * NULL, there are fewer parts (the same values up to rounding, in more time
 * where there are few rows); for one workspace size the results are
 * bit-identical from call to call.  A workspace serves one call at a time.
 * max_length: an upper bound of length that the caller knows (0: table_width
 * * N); it sizes the parts and limits nothing. */
typedef struct tl_attend_args {
    uint32_t struct_size;          /* sizeof(tl_attend_args) */
    int32_t n_heads;               /* a multiple of cache.n_kv_heads */
    tl_kv_view cache;
    int64_t n_tokens;              /* T >= 0 */
    const int64_t* q_offset;       /* [B+1]; NULL = one token each */
    const void* query;             /* [T][n_heads][D], strides in elements (multiples of 8) */
    int64_t query_token_stride, query_head_stride;
    float scale;                   /* finite, > 0 */
    int32_t window;                /* W >= 0; 0 = every earlier token */
    int32_t sinks;                 /* >= 0 */
    int32_t max_length;            /* 0 = unknown */
    void* out;                     /* [T][n_heads][D], contiguous, of the cache's dtype */
    float* lse;                    /* [T][n_heads]; NULL = not wanted */
    void* workspace;               /* nullable */
    uint64_t workspace_bytes;
    const int32_t* granted;        /* [n_seqs + 1], nullable (absent: a struct_size without it) */
} tl_attend_args;

tl_status tl_attend(const tl_attend_args* args, void* stream);
uint64_t tl_attend_workspace_bytes(const tl_attend_args* args);   /* 0 for arguments that tl_attend refuses */

/* ------------------------------------------------------------------------
 * The pool's pages.  ref[p] (int32 [n_pages]) counts the table entries that
 * hold page p; 0 = free.  Sequence slots are rows of page_table [n_slots]
 * [table_width]; the first ceil(length / N) entries of a row are its pages.
 * Free pages are taken in ascending order, so equal states give equal tables.
 * All state is the caller's, on the device; the calls change it in place in
 * stream order.  n_pages and n_slots are at most 2^31-1.
 *
 * Status per slot or fork, as the projection's queue decides: pages are given
 * in order, and an entry whose pages do not fit behind all earlier ones' gets
 * none (entries that need none are served all the same).
 * ---------------------------------------------------------------------- */
#define TL_PAGES_OK         0
#define TL_PAGES_NONE_FREE  1   /* the pool has too few free pages                    */
#define TL_PAGES_TABLE_FULL 2   /* more pages than table_width                        */
#define TL_PAGES_BAD        3   /* malformed entry (see each call)                    */

typedef struct tl_pages {
    uint32_t struct_size;          /* sizeof(tl_pages) */
    int32_t page_tokens;           /* N, 1 .. TL_MAX_BLOCK_TOKENS */
    int64_t n_pages;
    int64_t n_slots;
    int32_t table_width;
    int32_t reserved;
    int32_t* ref;                  /* [n_pages] */
    int32_t* page_table;           /* [n_slots][table_width] */
    int32_t* length;               /* [n_slots] */
    int32_t* granted;              /* [n_slots + 1], nullable (absent: a struct_size without it) */
} tl_pages;

/* int32 words that `work` of the calls below has to hold. */
uint64_t tl_pages_work_words(const tl_pages* pages);

/* Room for add[b] more tokens in every slot b, in slot order: the pages
 * behind its last one, ref 1, and length[b] += add[b].  TL_PAGES_BAD: add < 0
 * or length < 0.  Slots that are not served keep their length.
 * granted[b]: the tokens that slot b got since the last append, g, or -1 - g when
 * it was refused after that.  granted[n_slots]: 0 from here until tl_kv_append has
 * placed them (non-zero at first). */
tl_status tl_pages_extend(const tl_pages* pages, const int32_t* add, int32_t* status, int32_t* work, void* stream);

/* Fork i makes the empty slot child[i] a copy of parent[i]: it shares the full
 * pages (ref + 1) and gets a free page (ref 1) for a partly filled last one, which
 * tl_pages_copy has to fill from copy_src[i] to copy_dst[i] (both -1 when there
 * is nothing to copy).  So a page with room is only ever one sequence's.
 * Lengths are those before the call.  TL_PAGES_BAD: a slot out of range or of
 * negative length, child not empty, or an earlier fork's child; the child stays
 * empty then, as with TL_PAGES_NONE_FREE.  granted[child[i]] becomes 0 with the fork. */
tl_status tl_pages_fork(const tl_pages* pages, int64_t n_forks, const int32_t* parent, const int32_t* child,
                        int32_t* copy_src, int32_t* copy_dst, int32_t* status, int32_t* work, void* stream);

/* The slots leave: ref - 1 for each of their pages, length 0 (their table rows
 * are left as they are).  Slots out of range are ignored. */
tl_status tl_pages_free(const tl_pages* pages, int64_t n_free, const int32_t* slots, void* stream);

/* With L pages in use, pages L and up move to the free ones below L, both in
 * ascending order: copy_src[i] -> copy_dst[i] for i < *n_copies (each array has
 * room for n_pages / 2 entries), which tl_pages_copy does.  ref_out and
 * table_out (which may be pages->ref and pages->page_table) are the state
 * after that; entries past a slot's pages are copied, an entry that holds a
 * page nobody counts becomes -1. */
tl_status tl_pages_compact(const tl_pages* pages, int32_t* ref_out, int32_t* table_out, int32_t* copy_src,
                           int32_t* copy_dst, int32_t* n_copies, int32_t* work, void* stream);

/* Page copy_src[i] to page copy_dst[i] in every one of n_planes planes (the
 * layers' keys and values), for i < n_pairs, or i < *n_live (device, nullable;
 * at most n_pairs).  Page p of plane q is page_bytes bytes at pages + q *
 * plane_stride + p * page_stride (bytes; all multiples of 16, pages 16-byte
 * aligned).  Pairs with an index outside [0, n_pages) are skipped.  No page may
 * be both read and written. */
tl_status tl_pages_copy(void* pages, int64_t n_pages, int64_t page_bytes, int64_t page_stride, int32_t n_planes,
                        int64_t plane_stride, const int32_t* copy_src, const int32_t* copy_dst, int64_t n_pairs,
                        const int32_t* n_live, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TL_H */
