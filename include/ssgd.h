/*
 * ssgd.h -- C ABI of the Sketched-SGD compression step for NVIDIA B200 (sm_100a).
 *
 * One step of the paper's empirical training procedure (Algorithm 3, lines 5-13) over W workers
 * whose state lives, batched, on ONE GPU:
 *
 *   line 5   momentum                 u_w <- rho*u_w + g_w
 *   line 6   error accumulation       v_w <- v_w + u_w                       (the new u_w)
 *   line 7   Count Sketch of v_w      S_w[j][h_j(i)] += s_j(i) * v_w[i]      (Algorithm 4, update)
 *   line 8   aggregate                S = sum_w S_w                           (plain sum, see below)
 *   line 9   top-ncand by |estimate|  est[i] = median_j s_j(i)*S[j][h_j(i)]   (Algorithm 4, estimate)
 *   line 10  second round             xs[m] = sum_w v_w[cand[m]]
 *   line 11  k-sparse update          the k candidates with the largest |xs|
 *   line 13  masking / error reset    u_w[i] = v_w[i] = 0 at those k coordinates, every worker
 *
 * Conventions
 *  - Every call returns an int status: SSGD_OK (0) or a negative SSGD_E* code.  Nothing throws,
 *    aborts or traps.  Arguments are checked on the host before anything is launched.
 *  - "device" pointers are CUDA device pointers of the current device, owned by the caller.  The
 *    library allocates no device memory: all scratch is the caller's workspace (ssgd_bind).
 *  - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Stage calls and
 *    ssgd_step only enqueue work; they never synchronise.  Results are valid once the stream
 *    has reached that point.
 *  - Worker-major layout: g, u, v are [W][ld] fp32, row w at base + w*ld, only the first d entries
 *    of a row are read or written.  Bases must be 16-byte aligned and ld a multiple of 4
 *    (SSGD_EALIGN otherwise), ld >= d.
 *  - Hash family (fixed by the problem statement; Algorithm 4 line 2 leaves it open), p = 2^31-1:
 *        h_j(i) = ((a_j*i  + b_j ) mod p) mod c
 *        s_j(i) = 2*(((a'_j*i + b'_j) mod p) & 1) - 1
 *    with i the 0-based coordinate and j the 0-based row.  a_j, b_j, a'_j, b'_j come from `seed`:
 *    a 64-bit state s starts at seed; each draw does s += 0x9E3779B97F4A7C15, z = s,
 *    z = (z^(z>>30))*0xBF58476D1CE4E5B9, z = (z^(z>>27))*0x94D049BB133111EB, out = z^(z>>31);
 *    row j takes four draws in the order a, b, a', b' with a = 1 + out mod (p-1), b = out mod p.
 *  - The aggregate is the SUM of the workers' sketches and out_val is the SUM of the workers'
 *    values (Algorithm 3 line 10 stores the sum; the 1/W of line 8 does not change any selection).
 *  - Selections use the total order "larger magnitude first (fp32 bit pattern of |x|), then smaller
 *    coordinate index first", so they are unique given their inputs.
 *  - Inputs must be finite.  fp32 throughout; the only fused multiply-add is the momentum line.
 */
#ifndef SSGD_H
#define SSGD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SSGD_OK          0
#define SSGD_EINVAL     -1  /* bad shape, size, NULL pointer, ld < d, k > ncand, ncand > d, even r ... */
#define SSGD_EALIGN     -2  /* a base or ld not aligned as the call needs (the step: 16 bytes, ld % 4 == 0)  */
#define SSGD_ENOTBOUND  -3  /* ssgd_bind has not been called                                           */
#define SSGD_EWORKSPACE -4  /* workspace too small for the requested ncand                             */
#define SSGD_ECUDA      -5  /* a CUDA runtime call failed; ssgd_last_error gives its text              */
#define SSGD_EDEVICE    -6  /* a kernel recorded an error: bad index in a caller's list, or a wait gave up */
#define SSGD_ENOMEM     -7  /* host allocation failed                                                  */
#define SSGD_ETOOBIG    -8  /* beyond a fixed capacity: ssgd_exact_topk_static's scratch, SSGD_MAX_TOP      */
#define SSGD_EPENDING   -9  /* a deferred zero-out has not been applied yet: ssgd_flush first (or ssgd_unbind) */

#define SSGD_MAX_R 15

/* Insert variants of ssgd_step (ssgd_set_insert_mode) */
#define SSGD_INSERT_AUTO   0  /* SSGD_INSERT_TMA when W >= 144, else SSGD_INSERT_GLOBAL (measured)           */
#define SSGD_INSERT_GLOBAL 1  /* plain 128-bit loads; reductions straight into the L2-resident table    */
#define SSGD_INSERT_SMEM   2  /* per-block table in shared memory, flushed once; needs r*c*4 <= 200 KiB */
#define SSGD_INSERT_TMA    3  /* bulk-copy (TMA) + mbarrier pipeline; reductions into the L2 table      */

/* How ssgd_step evaluates Algorithm 3 line 9 (ssgd_set_prune_mode).  A median of r values reaches a magnitude
 * only if (r+1)/2 of them do, so with a threshold taken from a sample of the estimates most coordinates can be
 * ruled out from "is this bucket's magnitude above the threshold" alone.  ON: that test is precomputed as one bit
 * per bucket and kept in shared memory: all r*c bits at once if they fit; else one row (or one of up to four
 * slices of a row) per thread block, the r bits of every coordinate being combined afterwards; else OR-folded up
 * to 32 buckets per bit; otherwise as EARLY_EXIT.  EARLY_EXIT: the test is applied to the table values themselves and a coordinate stops reading
 * rows once it cannot pass.  OFF: every coordinate reads all r rows.  The candidates are identical in all modes.
 * AUTO is ON when d >= 2^21, ncand <= d/8 (below that the fixed costs outweigh the saving) and either the bitmap
 * fits as a whole or 5 <= r <= 9; else OFF.  Unless the bitmap fits as a whole, ON measures its density each step
 * and runs the EARLY_EXIT kernel instead when its bits would rule out too few coordinates. */
#define SSGD_PRUNE_AUTO 0
#define SSGD_PRUNE_OFF  1
#define SSGD_PRUNE_ON   2
#define SSGD_PRUNE_EARLY_EXIT 3
/* FUSED: lines 9-13 run as ONE cooperative kernel (dense estimates, exact radix select and ordered candidate emit
 * behind grid barriers, the second round where a candidate is emitted, the final top-k and line 13 by the last
 * block), for problems so small that a chain of short
 * launches costs more than the work: needs d <= 2^22 and ncand <= 16384 (SSGD_EINVAL from ssgd_step otherwise).
 * AUTO takes this path for d <= 2^21 when it applies.  The results are those of the other modes. */
#define SSGD_PRUNE_FUSED 4

typedef struct ssgd_ctx ssgd_ctx; /* opaque host object; holds no device memory */

/* Algorithm 4 init(r, c) plus the shape of Algorithm 3: d coordinates, r rows (odd, 1..15), c columns,
 * k final sparsity, W workers; 1 <= d < 2^31-1, 1 <= c < 2^31-1, 1 <= k <= d, W >= 1.  Host only. */
int ssgd_create(ssgd_ctx** out, int64_t d, int32_t r, int64_t c, int64_t k, int32_t W, uint64_t seed);
/* Frees the host object.  While a deferred zero-out of the last ssgd_step is still pending (see
 * ssgd_set_zero_mode) the bound u and v do not hold Algorithm 3 line 13's zeros yet and the marks live only in
 * the workspace, so the call refuses with SSGD_EPENDING and leaves the context alive: call ssgd_flush first, or
 * ssgd_unbind to give the marks up on purpose.  (It does not write the zeros itself because it cannot know
 * that the caller's buffers still exist.) */
int ssgd_destroy(ssgd_ctx* ctx);

/* The 4r hash parameters, row j at out4r[4j..4j+3] = a_j, b_j, a'_j, b'_j (host memory). */
int ssgd_get_hash_params(const ssgd_ctx* ctx, uint32_t* out4r);
/* Replace them (for tests): a, a' in [1, p-1], b, b' in [0, p-1]. */
int ssgd_set_hash_params(ssgd_ctx* ctx, const uint32_t* in4r);
int ssgd_set_insert_mode(ssgd_ctx* ctx, int32_t mode);
int ssgd_set_prune_mode(ssgd_ctx* ctx, int32_t mode);
/* When ssgd_step applies Algorithm 3 line 13 (u, v <- 0 at the k chosen coordinates).
 * DEFERRED (default): ssgd_step only marks the chosen coordinates in a d-bit map inside the workspace; the NEXT
 * ssgd_step reads marked coordinates of u and v as +0 inside the kernel that streams all of u and v anyway, so
 * the zero-out costs no scattered writes.  Until then the memory of u and v still holds the old values at those
 * coordinates: call ssgd_flush before reading u or v yourself.  The library's own entry points that read u or v
 * (ssgd_sketch_accumulate, ssgd_exact_topk, ssgd_heavymix) flush first; ssgd_exact_topk_static has no context
 * and cannot.  Every result (chosen coordinates, values, the state after a flush) is identical in both modes.
 * The pending marks are state of the method that lives in the workspace: to checkpoint, call ssgd_flush and
 * save u and v; ssgd_bind and ssgd_destroy refuse (SSGD_EPENDING) while marks are pending.
 * EAGER: ssgd_step writes the zeros before it returns control to the stream's next operation. */
#define SSGD_ZERO_DEFERRED 0
#define SSGD_ZERO_EAGER    1
int ssgd_set_zero_mode(ssgd_ctx* ctx, int32_t mode);
/* Limit, in nanoseconds (>= 1000; default 2e9), of every wait inside a kernel: the grid barriers of the FUSED tail
 * and the pipeline barriers of the bulk-copy insert kernel.  A wait that runs out makes its kernel record an
 * error and return; ssgd_status then reports SSGD_EDEVICE once, results of that step are undefined, and the
 * context stays usable. */
int ssgd_set_wait_limit_ns(ssgd_ctx* ctx, int64_t ns);
/* Test hook: thread block (block_plus_one - 1) of those kernels leaves without ever arriving at its barriers, so
 * that the others' waits run out (nothing hangs, nothing faults); 0 switches the hook off.  -1: ssgd_step behaves as
 * if the device had refused the cooperative launch of the FUSED tail (which happens when it cannot hold one thread
 * block per SM at once, e.g. with SMs taken by another context): under SSGD_PRUNE_AUTO the step then takes the chain
 * of ordinary launches, and so do the following steps; under SSGD_PRUNE_FUSED it returns SSGD_ECUDA. */
int ssgd_test_withhold_block(ssgd_ctx* ctx, int32_t block_plus_one);
/* Applies a deferred zero-out to u and v now (device pointers bound by ssgd_bind), on `stream`.  Cheap when
 * nothing is pending (one pass over d/8 bytes).  It always launches: the marks may come from a replayed CUDA
 * graph, which the host side of the context does not see. */
int ssgd_flush(ssgd_ctx* ctx, void* stream);
/* For tables too large to stay in L2 next to the streamed g, u, v: let the streaming kernel insert only as
 * many rows as fit in `bytes` and insert the remaining rows from the per-coordinate sums in follow-up
 * launches of at most `bytes` of table each (plain-load insert variant only; 0 = never split; default 24 MiB,
 * which leaves tables up to that size untouched). */
int ssgd_set_insert_split(ssgd_ctx* ctx, int64_t bytes);
/* Cache operator of the plain-load accumulate+insert kernel's reads of g, u, v (ssgd_step with
 * SSGD_INSERT_GLOBAL).  AUTO = L2_ONLY (ld.global.cg: not kept in L1, normal priority in L2; the table's lines are
 * protected by the evict-last policy of the reductions).  EVICT_FIRST: ld.global.cs.  The result of a step does
 * not depend on it. */
#define SSGD_STREAM_AUTO        0
#define SSGD_STREAM_EVICT_FIRST 1
#define SSGD_STREAM_L2_ONLY     2
int ssgd_set_stream_loads(ssgd_ctx* ctx, int32_t mode);
/* Opt-in: reserve part of L2 for the sketch table while the accumulate+insert kernel streams g, u, v past it
 * (cudaLimitPersistingL2CacheSize of this process's CUDA context is raised to the table size, capped by the
 * device; the launches then carry an access-policy window over the table).  Off by default because the limit
 * is shared with everything else the process runs on that device.  enable = 0 stops attaching the window. */
int ssgd_set_table_persistence(ssgd_ctx* ctx, int32_t enable);
/* Diagnostics of the last ssgd_step's pruned path (waits for the stream), five values: out[0] != 0 if the
 * sampled threshold kept fewer than ncand coordinates and the pass was redone without pruning, out[1] = number
 * of coordinates on the survivor list, out[2] = the prune threshold as a histogram-bin index (0: nothing
 * pruned), out[3] = 1 if the bucket bitmap was too dense and the first pass read the table instead,
 * out[4] = set bits of the bitmap that was measured (the unfolded one if it is used row by row, else the folded
 * one; 0 if the bitmap fits shared memory as a whole and is not measured). */
int ssgd_step_used_fallback(ssgd_ctx* ctx, void* stream, int32_t* out5);
/* Diagnostics of the last ssgd_step that took the FUSED tail (waits for the stream): nanoseconds since the tail
 * kernel's first thread block started, at 12 points -- [0] start, [1] table rows copied to shared memory (if any),
 * [2] its estimates done, [3]-[5] past the first three grid barriers (the digits of the threshold), [11] past the
 * fourth (segment counts complete), all of thread block 0; of the block that finishes the step alone: [6] it knows
 * it is the last (candidates and their sums are in place), [7], [8] candidates loaded, [9] final threshold known,
 * [10] end.  -1 where no stamp was taken. */
int ssgd_tail_trace(ssgd_ctx* ctx, void* stream, int64_t* out12);
/* For tests and diagnostics: the rank (from the top) in the sample's histogram that sets the prune threshold;
 * 0 = derive it from ncand (mean + 6 sigma + 16).  A rank of 1 puts the threshold at the largest sampled
 * estimate, which forces the unpruned rerun. */
int ssgd_set_prune_sample_rank(ssgd_ctx* ctx, int64_t rank);

/* Bytes of device scratch needed to run steps with up to ncand_max candidates (host only). */
int ssgd_workspace_bytes(const ssgd_ctx* ctx, int64_t ncand_max, size_t* out_bytes);

/* Attach the caller-owned worker state u, v ([W][ld] fp32, device; Algorithm 3 line 1 wants them
 * zero before the first step) and the caller-owned workspace (device, 256-byte aligned, at least
 * ssgd_workspace_bytes(ncand_max)).  The buffers must stay valid while the context uses them.  Rebinding a
 * context whose last step's zero-out is still pending is refused with SSGD_EPENDING (see ssgd_destroy). */
int ssgd_bind(ssgd_ctx* ctx, float* u, float* v, int64_t ld, void* workspace, size_t workspace_bytes,
              int64_t ncand_max);
/* Detaches u, v and the workspace.  A pending deferred zero-out is DISCARDED (the previously bound u and v keep
 * their old values at the last step's k coordinates): the explicit way out of SSGD_EPENDING for a caller who no
 * longer wants that state.  Touches no device memory. */
int ssgd_unbind(ssgd_ctx* ctx);

/* Algorithm 3 lines 5-7 (Algorithm 4 update): updates the bound u, v from g ([W][ld_g] fp32, device,
 * read only) and writes each worker's own sketch to tables[w] ([W][r][c] fp32, device; zeroed by the
 * call, then filled with reductions, so bucket sums are order-dependent in the last bits). */
int ssgd_sketch_accumulate(ssgd_ctx* ctx, const float* g, int64_t ld_g, float rho, float* tables,
                           void* stream);

/* How ssgd_sketch_accumulate walks the W x d worker-coordinates.  COORDINATE_MAJOR: one launch, a thread owns a
 * group of coordinates and visits every worker (hashes computed once per coordinate; reductions scatter over all
 * W tables at once).  WORKER_MAJOR: one launch per worker, so that only that worker's r x c table receives
 * reductions and stays L2-resident meanwhile (hashes recomputed per worker).  AUTO: WORKER_MAJOR once the W
 * tables together exceed 32 MiB.  The results are the same up to the order of the reductions. */
#define SSGD_SCHED_AUTO             0
#define SSGD_SCHED_COORDINATE_MAJOR 1
#define SSGD_SCHED_WORKER_MAJOR     2
int ssgd_set_accumulate_schedule(ssgd_ctx* ctx, int32_t mode);

/* Algorithm 3 line 8 (mergeability, Section 3): merged[j][b] = sum over w = 0..W-1, in that order,
 * of tables[w][j][b].  merged is [r][c] fp32, device. */
int ssgd_sketch_merge(ssgd_ctx* ctx, const float* tables, float* merged, void* stream);

/* 16-bit sketches (Section 6: quantising sketches to 16 bits).  ssgd_sketch_quantize16 rounds the W per-worker
 * tables ([W][r][c] fp32, device) to a 16-bit format, round-to-nearest-even -- SSGD_FMT_F16: IEEE binary16,
 * magnitudes beyond 65504 saturate; SSGD_FMT_BF16: bfloat16 -- into q16 ([W][r][c] uint16, device): what each
 * worker would transmit.  ssgd_sketch_merge16 is the server side: merged[j][b] = sum over w = 0..W-1, in that
 * order, in fp32, of the decoded q16[w][j][b].  The rest of the pipeline runs on `merged` unchanged. */
#define SSGD_FMT_F16  0
#define SSGD_FMT_BF16 1
#define SSGD_FMT_F32  2  /* the training operators below */
#define SSGD_FMT_E4M3 3  /* ssgd_adamw_step's 8-bit states */
int ssgd_sketch_quantize16(ssgd_ctx* ctx, const float* tables, int32_t fmt, uint16_t* q16, void* stream);
int ssgd_sketch_merge16(ssgd_ctx* ctx, const uint16_t* q16, int32_t fmt, float* merged, void* stream);

/* Algorithm 3 line 9 (Algorithm 4 estimate for every coordinate, Section 5.2): computes est[i] for
 * all i < d from merged ([r][c] fp32, device) and writes the ncand coordinates with the largest
 * |est| to cand_idx ([ncand] int32, device), in ASCENDING coordinate order.  cand_est ([ncand] fp32)
 * and est_all ([d] fp32, 16-byte aligned) are optional device outputs (NULL to skip).  k <= ncand <= d. */
int ssgd_unsketch_candidates(ssgd_ctx* ctx, const float* merged, int64_t ncand, int32_t* cand_idx,
                             float* cand_est, float* est_all, void* stream);

/* Algorithm 3 lines 10, 11 and 13: sums the bound v over workers at each candidate (fp64, w = 0..W-1),
 * keeps the k largest by |sum| (ties: earlier position in cand_idx, which is the smaller coordinate
 * when cand_idx is ascending), writes them to out_idx/out_val ([k], device, in cand_idx order), and
 * then sets u and v to +0.0f at those k coordinates in every worker.  Entries of cand_idx must be
 * distinct and in [0, d); an out-of-range entry is skipped and reported by ssgd_status. */
int ssgd_exact_topk(ssgd_ctx* ctx, const int32_t* cand_idx, int64_t ncand, int32_t* out_idx,
                    float* out_val, void* stream);

/* Algorithm 3 lines 5-13 in one call: the stages above, with the workers' values summed before the
 * insert (sum_w S(v_w) = S(sum_w v_w), Section 3), so no per-worker table is materialised.
 * The same kernel keeps each coordinate's sum over the workers (fp64, worker order, rounded once), so line 10
 * reads one number per candidate instead of W values of v; the result is bit-identical to ssgd_exact_topk's.
 * out_idx/out_val: [k] device outputs, ascending coordinate order.  Line 13 is applied as ssgd_set_zero_mode
 * says: by default it is deferred into the next ssgd_step (or ssgd_flush). */
int ssgd_step(ssgd_ctx* ctx, const float* g, int64_t ld_g, float rho, int64_t ncand,
              int32_t* out_idx, float* out_val, void* stream);

/* Algorithm 1 (HEAVYMIX), the selection rule of the paper's analysis, on a merged [r][c] table (device):
 *   line 1  l2 = median over rows of the row's sum of squared counters (fp64)
 *   line 3  H = { i : est_i^2 >= l2 / k }, est the median-of-r estimate, compared in fp64
 *   line 4  Top_k = H plus a uniformly random (k - |H|)-subset of the other coordinates: every coordinate has
 *           a 30-bit priority mixed from (fill_seed, i) -- z = fill_seed + (i+1)*0x9E3779B97F4A7C15,
 *           z = (z^(z>>30))*0xBF58476D1CE4E5B9, z = (z^(z>>27))*0x94D049BB133111EB, z ^= z>>31, priority = z>>34
 *           -- and the non-heavy coordinates with the largest priorities are taken (ties: smaller index).
 *           Should more than k coordinates be heavy (outside the paper's guarantee), the k heavy coordinates
 *           with the largest |est| are kept (fp32 bit pattern of the magnitude, ties: smaller index) and
 *           nothing else.
 *   line 5  out_val[t] = sum over the workers of the bound v at out_idx[t] (fp64, worker order).
 * out_idx / out_val: [k] device outputs, ascending coordinate order.  l2_out (device double) and nheavy_out
 * (device int32) are optional.  The bound state is read, not modified (a deferred zero-out is applied first).
 * Asynchronous on `stream`. */
int ssgd_heavymix(ssgd_ctx* ctx, const float* merged, uint64_t fill_seed, int32_t* out_idx, float* out_val,
                  double* l2_out, int32_t* nheavy_out, void* stream);

/* The same step for a caller whose gradients and results live in HOST memory: copies g_host
 * ([W][ld_g] fp32; pinned memory makes the copy asynchronous) into g_stage (device, [W][ld_g]),
 * runs ssgd_step, copies the k results back to out_idx_host/out_val_host and waits for the stream. */
int ssgd_step_host(ssgd_ctx* ctx, const float* g_host, int64_t ld_g, float rho, int64_t ncand,
                   float* g_stage, int32_t* out_idx_host, float* out_val_host, void* stream);

/* Device pointers into the workspace holding, after ssgd_step, the merged [r][c] table, est[d] and
 * the candidate list [ncand] (for tests and diagnostics).  Any of the outputs may be NULL.  est[d] is
 * only filled when the step ran without pruning (or fell back to the dense path). */
int ssgd_step_buffers(const ssgd_ctx* ctx, const float** merged, const float** est,
                      const int32_t** cand_idx, const float** cand_xs);

/* h_j(i), s_j(i) for n coordinates idx[n] (device int32) -> h_out, s_out ([r][n] int32, device).
 * The same device functions the step uses (Algorithm 4 lines 2, 6, 11); for bit-exactness checks. */
int ssgd_hashes(ssgd_ctx* ctx, const int32_t* idx, int64_t n, int32_t* h_out, int32_t* s_out,
                void* stream);

/* Second round and final top-k WITHOUT a workspace.  (The paper has no counterpart: this exists for
 * the way the library gets embedded, not for the method.)
 *
 * Who needs it: code that is handed gradient and state buffers but may not allocate device memory
 * itself -- a compression hook called from inside a trainer whose caching allocator owns the whole
 * GPU (a raw cudaMalloc there can fail, and it stalls every stream of the device while it runs), or a
 * caller on a latency-critical path that must not trigger allocation at all.  Such a caller cannot
 * provide the workspace that ssgd_bind asks for, so this entry point keeps its scratch (second-round
 * sums, radix histograms, chunk counters) in a fixed array of SSGD_STATIC_SCRATCH_BYTES (1.06 MiB)
 * that is part of the library image: every GPU that loads the library holds that much until the
 * process exits.  The call itself allocates nothing, on the host or on the device.
 *
 * What it computes: Algorithm 3 lines 10-11 exactly as ssgd_exact_topk does -- xs[m] = sum over
 * w = 0..W-1 of v[w][cand_idx[m]] (fp64, that order), then the k entries with the largest |xs|, ties
 * to the earlier position -- written to out_idx/out_val ([k], device) in cand_idx order.  It does NOT
 * zero any state (line 13 stays with the caller) and needs no context: v ([W][ld] fp32, device),
 * cand_idx ([ncand] int32, device, distinct, in [0, d); out-of-range entries count as zero) and the
 * sizes are passed directly.  k <= ncand <= min(d, SSGD_STATIC_MAX_NCAND); a larger ncand is refused
 * with SSGD_ETOOBIG before anything is launched.
 *
 * Sharing: all calls on one GPU use the same array, and it still holds the previous call's data.
 * Each call first clears the parts that must start at zero, in stream order.  Two calls whose work
 * can overlap on the GPU (different streams without an ordering between them, or different host
 * threads doing so) race on the array and give wrong results: keep calls on one device ordered.
 * The first call on each device looks up the array's device address (cudaGetSymbolAddress, with that
 * device current); make that first call before starting any stream capture.  Asynchronous on
 * `stream` like the other stage calls. */
#define SSGD_STATIC_MAX_NCAND     262144
#define SSGD_STATIC_SCRATCH_BYTES 1114112
int ssgd_exact_topk_static(const float* v, int64_t ld, int32_t W, int64_t d, const int32_t* cand_idx,
                           int64_t ncand, int64_t k, int32_t* out_idx, float* out_val, void* stream);

/* Optional per-stage timing of ssgd_step with CUDA events recorded on the caller's stream (up to 256
 * steps between collections).  Stages: 0 = the accumulate+insert kernel, 1 = the unsketch kernel,
 * 2 = candidate selection, 3 = second round + final top-k + zero-out.  ssgd_get_stage_times waits for
 * the stream, writes the summed milliseconds per stage to ms_out[SSGD_NSTAGES] and the number of steps
 * they cover to steps_out (host memory), and starts a new collection. */
#define SSGD_NSTAGES 4
int ssgd_set_timing(ssgd_ctx* ctx, int32_t enable);
int ssgd_get_stage_times(ssgd_ctx* ctx, void* stream, double* ms_out, int64_t* steps_out);

/* Number of kernels (and memset nodes) the library has launched through this context so far. */
int ssgd_launch_count(const ssgd_ctx* ctx, int64_t* out);

/* Waits for the stream, then returns SSGD_EDEVICE if a kernel recorded an error since the last call
 * (the flag is cleared), SSGD_ECUDA if the stream reports a CUDA error, else SSGD_OK. */
int ssgd_status(ssgd_ctx* ctx, void* stream);

/* ---- operators of the training step around the compression ------------------------------------------------------
 *
 * The gradient that ssgd_step compresses comes out of a model's layers and loss, and the parameters that are not
 * sketched (Section 5 of the paper leaves bias terms uncompressed) need an ordinary optimizer step.  These entry
 * points have no context: everything they read or write is an argument.  They allocate nothing, check their arguments
 * before anything is launched, and only enqueue work on `stream`, so they can be captured in a CUDA graph.  A graph repeats the
 * call as it was captured: of ssgd_adamw_step that includes lr, the step's number in its bias corrections and the seed, so a
 * replayed step has the same dither every time.  Capture it anew for every step (or leave it out of the graph).
 *
 * Element formats are SSGD_FMT_*; all arithmetic is fp32, results are rounded to nearest even once.  Bases need the
 * alignment of their element type only (SSGD_EALIGN); rows may have any stride ld >= n (elements).  Bases and
 * strides that are multiples of 16 bytes are fastest.  Values may be anything: infinities and NaN follow the formulas.
 */

/* Layer norm over the last dimension of x [rows][n] (any of the three formats):
 *   mean = 1/n sum x,  rstd = (1/n sum (x - mean)^2 + eps)^-1/2,  y = (x - mean) rstd w + b
 * w, b: [n] in fmt_w, which is SSGD_FMT_F32 or fmt_x; either may be NULL (1 and 0).  y: [rows][n] in fmt_x, may be x
 * itself (same ld).  stats: [2][rows] fp32, mean then rstd: what the backward pass wants.  1 <= n <= 2^24, rows >= 0. */
int ssgd_layer_norm(const void* x, int64_t ld_x, int32_t fmt_x, const void* w, const void* b, int32_t fmt_w,
                    int64_t rows, int64_t n, float eps, void* y, int64_t ld_y, float* stats, void* stream);
/* Its gradient.  With h = (x - mean) rstd and a = dy w:
 *   dx = rstd (a - 1/n sum a - h 1/n sum a h)      [rows][n] in fmt_x; may be dy itself (same ld)
 *   dw = sum over rows of dy h,  db = sum over rows of dy      [n] fp32 (so they can be a piece of a row of g); either
 *        may be NULL; accumulate != 0 adds to what is there
 * The sums over rows are added in a fixed order.  workspace: device memory of at least
 * ssgd_layer_norm_backward_workspace(rows, n) bytes, 16-byte aligned, free again once the stream has passed. */
int ssgd_layer_norm_backward_workspace(int64_t rows, int64_t n, size_t* out_bytes);
int ssgd_layer_norm_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, int32_t fmt_x, const void* w,
                             int32_t fmt_w, const float* stats, int64_t rows, int64_t n, void* dx, int64_t ld_dx,
                             float* dw, float* db, int32_t accumulate, void* workspace, size_t workspace_bytes,
                             void* stream);

/* Log probabilities of given tokens.  For each row of logits [rows][vocab], z = scale * logits (scale > 0, e.g. 1 /
 * temperature), lse = log sum e^z, p = e^(z - lse):
 *   stats [3][rows] fp32   logp = z[id] - lse;  entropy = -sum p log p;  lse
 *   top_idx, top_logp [rows][top]   the `top` (0 .. SSGD_MAX_TOP) largest logits, larger first, equal ones by smaller
 *                                   index (NaN counts as the largest), and their log probabilities
 * ids: [rows] of 4 or 8 bytes each (ids_bytes).  An id outside [0, vocab) is ignored: its logp is 0 and has no gradient.
 * A logit of -inf has probability 0.  A row of nothing else has lse = -inf, entropy 0 and every log probability -inf (of its
 * gradient, with p = 0, only the terms at id and top_idx themselves are left).  Finite logits may be as far from zero as they
 * like.  A NaN or +inf makes its row's statistics NaN.  1 <= vocab <= 2^27. */
#define SSGD_MAX_TOP 32
int ssgd_token_logprobs(const void* logits, int64_t ld, int32_t fmt, const void* ids, int32_t ids_bytes, int64_t rows,
                        int64_t vocab, float scale, int32_t top, float* stats, int32_t* top_idx, float* top_logp,
                        void* stream);
/* The gradient with respect to the logits of sum(d_logp logp) + sum(d_entropy entropy) + sum(d_top top_logp):
 *   dlogits_j = scale (d_logp [j = id] + sum_m d_top_m [j = top_idx_m] - p_j (d_logp + sum_m d_top_m + d_entropy (log p_j + entropy)))
 * with p_j = e^(z_j - lse), at most 1.  lse, entropy: [rows], as the forward pass wrote them.  d_logp, d_entropy: [rows], either may be NULL (0).  top_idx, d_top:
 * [rows][top].  A top_idx outside [0, vocab) adds to the sum only.  dlogits: [rows][vocab] in fmt; may be logits itself
 * (same ld). */
int ssgd_token_logprobs_backward(const void* logits, int64_t ld, int32_t fmt, const void* ids, int32_t ids_bytes,
                                 int64_t rows, int64_t vocab, float scale, const float* lse, const float* entropy,
                                 const float* d_logp, const float* d_entropy, int32_t top, const int32_t* top_idx,
                                 const float* d_top, void* dlogits, int64_t ld_d, void* stream);

/* One AdamW step (decoupled weight decay) over `count` tensors, each contiguous, in one launch per 384 tensors:
 *   g <- g * grad_scale (device fp32 scalar, NULL: 1)
 *   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2
 *   p <- p (1 - lr weight_decay) - lr / (1 - b1^step) * m / (sqrt(v) / sqrt(1 - b2^step) + eps),   step = 1, 2, ...
 * p: SSGD_FMT_F32 or SSGD_FMT_BF16.  g: fp32, binary16 or bfloat16.  copy: NULL, or (fp32 p only) a copy of the new p
 * in fmt_copy (SSGD_FMT_BF16 or SSGD_FMT_F16).  No two of these buffers may overlap.
 * States, fmt_state: SSGD_FMT_F32, m and v fp32 [n], scales unused; or SSGD_FMT_E4M3, one byte per element: every
 * SSGD_ADAMW_BLOCK consecutive elements share an fp32 scale (m_scale, v_scale: [ceil(n / SSGD_ADAMW_BLOCK)]), m stands
 * for code * m_scale and v for (code * v_scale)^2.  Zero codes and scales are the initial state.  Every operation on them is
 * rounded to fp32 by itself, in this order, so that equal states give equal states on any machine:
 *   m = (code m_scale) b1 + g (1 - b1);   r = code v_scale,  v = (r r) b2 + (g g) (1 - b2),  x = |m| or sqrt(v);
 *   with a the block's largest x, the new scale is a (1 / 448), y = x ((1 / a) 448), and the new code the multiple
 *   floor(y / unit + u) of the e4m3 numbers' unit at y; u = 1/2, or the dither (see stochastic).
 * A block whose a is below 2^-100 gets scale 0.  A positive sqrt(v) gets no smaller code than the least positive one.  A value that
 * is not finite is stored as NaN and left out of a.
 * stochastic != 0: e4m3 states and bfloat16 parameters are rounded up or down with the probability that makes them
 * right on average, by a hash of (seed, the tensor's place in the list, the element's index): give every step another
 * seed.  stochastic == 0: to nearest. */
#define SSGD_ADAMW_BLOCK 256
typedef struct {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    void* copy;
    int64_t n;
} ssgd_adamw_tensor;
int ssgd_adamw_step(const ssgd_adamw_tensor* tensors, int32_t count, int32_t fmt_p, int32_t fmt_g, int32_t fmt_state,
                    int32_t fmt_copy, double lr, double beta1, double beta2, double eps, double weight_decay,
                    int64_t step, const float* grad_scale, int32_t stochastic, uint64_t seed, void* stream);

/* The clipped policy loss of sampled tokens, and its gradient, in one pass over the logits.  For each row of logits [rows][vocab], z, lse,
 * p, logp = z[id] - lse and the entropy H as above:
 *   r = e^(logp - old_logp),  kept = A >= 0 ? min(r, 1 + clip_high) : max(r, 1 - clip_low),  A = advantages[row]
 *   q = ref_logp - logp,  K = e^q - 1 - q                     (0 without ref_logp)
 *   loss = w (-kept A + kl K - entropy H),   w = weights[row] (NULL: 1; a mean is a matter of the weights)
 *   c = (kept = r ? -A r : 0) - kl (e^q - 1)
 *   dlogits_j = w scale (c [j = id] - c p_j + entropy p_j (log p_j + H)), the gradient of the sum of the losses
 * stats [5][rows] fp32: loss, logp, H, K, r.  dlogits: [rows][vocab] in fmt, may be logits itself (same ld); NULL: not wanted.
 * A row of weight 0, or with an id outside [0, vocab), has statistics and gradient 0, whatever its logits are: they are not read.
 * old_logp, advantages, ref_logp, weights: [rows] fp32.  0 <= clip_low <= 1, 0 <= clip_high (infinity: no clipping), kl >= 0 (needs
 * ref_logp unless 0); entropy may be negative.  -inf logits, rows of nothing else, far logits and NaN: as for ssgd_token_logprobs. */
int ssgd_policy_loss(const void* logits, int64_t ld, int32_t fmt, const void* ids, int32_t ids_bytes, int64_t rows, int64_t vocab,
                     float scale, const float* old_logp, const float* advantages, const float* ref_logp, const float* weights,
                     float clip_low, float clip_high, float kl, float entropy, float* stats, void* dlogits, int64_t ld_d,
                     void* stream);

/* The preference loss of pairs of token sequences.  Sequence s is tokens [starts[s], starts[s + 1]) (starts: [2 pairs + 1] ascending, of 4 or
 * 8 bytes each; sequences may be empty); pair p is sequence 2 p, the preferred one, and 2 p + 1.  With
 *   D_s = sum of (logp - ref_logp) over the sequence, divided by its length if average != 0,   x = beta (D_2p - D_2p+1)
 * SSGD_PREFERENCE_SIGMOID   l = -(1 - e) log sigmoid(x) - e log sigmoid(-x),  e = label_smoothing, 0 .. 0.5
 * SSGD_PREFERENCE_IPO       l = ((x - 1/2) / beta)^2
 * SSGD_PREFERENCE_HINGE     l = max(0, 1 - x)
 *   loss [pairs] = weights l;  rewards [2][pairs] = beta D, of the preferred sequences and of the others;
 *   d_logp [tokens] (NULL: not wanted) = the gradient of the sum of the losses; 0 for tokens of no sequence
 * logp, ref_logp (NULL: 0), d_logp: [tokens] fp32; weights [pairs] fp32 (NULL: 1; a pair of weight 0 has loss and gradient 0 whatever
 * its tokens hold).  Differences and sums hold 48 bits or more and the range of 64-bit numbers, in an order that depends on nothing but the starts.  starts outside [0, tokens] count as the
 * nearest of these; where they do not ascend, the results of the pairs concerned are unspecified.
 * d_logp may be logp or ref_logp itself.  workspace: device memory of at least ssgd_preference_loss_workspace(tokens, pairs) bytes, 8-byte
 * aligned, free again once the stream has passed.  tokens <= 2^40, pairs <= 2^30. */
#define SSGD_PREFERENCE_SIGMOID 0
#define SSGD_PREFERENCE_IPO     1
#define SSGD_PREFERENCE_HINGE   2
int ssgd_preference_loss_workspace(int64_t tokens, int64_t pairs, size_t* out_bytes);
int ssgd_preference_loss(const float* logp, const float* ref_logp, int64_t tokens, const void* starts, int32_t starts_bytes, int64_t pairs,
                         const float* weights, int32_t kind, float beta, float label_smoothing, int32_t average, float* loss,
                         float* rewards, float* d_logp, void* workspace, size_t workspace_bytes, void* stream);

/* Orthogonalised matrices.  With u a matrix and |u| the root of the sum of its squares, x_0 = u / (|u| + eps), and `steps` times
 *   A = x x',  x <- a x + (b A + c A A) x          (rows <= cols; otherwise A = x' x and x <- a x + x (b A + c A A))
 * which applies the polynomial a s + b s^3 + c s^5 to the singular values; (3.4445, -4.7750, 2.0315) brings them near 1 in 5 steps.
 * The products are of fp16 numbers with fp32 sums.  products = 3: every matrix is a sum of two fp16 numbers, and results are about as exact as
 * in fp32 (measured: off by 4e-7 to 7e-6 of their norm, the same iteration in fp32 by 4e-7 to 1.5e-5; of a shorter side up to 16 beside a
 * longer one over 150 up to 4 times as far as fp32); 1: one number in the operands of products, two in x itself: the result is off by about
 * 1e-3 of its norm (1.5e-3 at most, but for matrices of less than 512 numbers, whose roundings do not average out: up to 7e-3);
 * 0: 1 for results in bfloat16, otherwise 3.
 * A matrix of zeros stays one (0 / 0 with eps = 0 is NaN), and numbers of x_0 below 2^-35 count as zero; infinities and NaN spread
 * over their matrix.  Polynomials that take anything in [0, 1] beyond 4 on the way, or beyond 8 at the end, are refused
 * (SSGD_EINVAL).  1 <= steps <= 32; rows,
 * cols <= 2^20, rows * cols <= 2^32, the shorter side <= 32768 (SSGD_ETOOBIG).  Matrices without elements are left out. */
typedef struct {
    void* out;        /* ssgd_orthogonalize: the result, may be `in` itself (same ld); ssgd_muon_step: the parameter */
    const void* in;   /* the matrix, or the gradient */
    float* m;         /* ssgd_muon_step: momentum, [rows][cols]; otherwise unused */
    int64_t ld_out, ld_in;
    int64_t rows, cols;
    double scale;     /* ssgd_muon_step: factor of lr for this matrix */
} ssgd_matrix;
/* Device memory that the two below need: 8 bytes per element of the matrices, twice (products 1) or four times (3) 2 bytes per element
 * of A, where both sides count as rounded up to 64, and a little; none for matrices of up to 128 x 256 or 256 x 128.  More than 224 matrices
 * or 2^27 elements (rounded up likewise) are worked off in groups, each in the same memory: 1.1 GB, and as much again at most for A (square
 * matrices, products 3), unless a single matrix needs more.  Free again once the stream has passed; its contents mean nothing.  16-byte
 * aligned. */
int ssgd_orthogonalize_workspace(const ssgd_matrix* matrices, int32_t count, int32_t fmt_out, int32_t products, size_t* out_bytes);
/* out <- the orthogonalised `in`, for each matrix; both in fmt. */
int ssgd_orthogonalize(const ssgd_matrix* matrices, int32_t count, int32_t fmt, int32_t products, int32_t steps, double a, double b,
                       double c, double eps, void* workspace, size_t workspace_bytes, void* stream);
/* One step of an optimizer for matrices, over `count` of them:
 *   g <- g * grad_scale (device fp32 scalar, NULL: 1),  m <- momentum m + (1 - momentum) g
 *   u = momentum m + (1 - momentum) g (nesterov != 0) or m,  p <- p (1 - lr weight_decay) - lr scale O(u)
 * with O(u) the orthogonalised u.  p: SSGD_FMT_F32 or SSGD_FMT_BF16; g: any of the three formats.  No two p or m may overlap. */
int ssgd_muon_step(const ssgd_matrix* matrices, int32_t count, int32_t fmt_p, int32_t fmt_g, int32_t products, double lr, double momentum,
                   int32_t nesterov, double weight_decay, int32_t steps, double a, double b, double c, double eps, const float* grad_scale,
                   void* workspace, size_t workspace_bytes, void* stream);
/* Waits for the stream; SSGD_EDEVICE if a wait inside a kernel of the training operators has run out on this device since the last
 * call (what that call wrote is then worthless), SSGD_ECUDA if the stream reports an error, else SSGD_OK.  Not while capturing. */
int ssgd_train_ops_status(void* stream);
/* Test hook: a kernel of which one warp waits at a barrier as those kernels do, half of its lanes for limit_ns (1000 .. 1e9), the others until
 * another warp arrives there, after the first have given up.  told: 32 numbers on the device, whether each lane was told that the wait
 * succeeded.  ssgd_train_ops_status reports it. */
int ssgd_test_run_out(int64_t limit_ns, int32_t* told, void* stream);

const char* ssgd_strerror(int code);
const char* ssgd_last_error(const ssgd_ctx* ctx); /* text of the last CUDA error seen, or "" */

#ifdef __cplusplus
}
#endif
#endif
