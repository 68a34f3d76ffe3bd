/*
 * stagefrontier.h - C ABI of libstagefrontier, synchronization-aware frontier
 * accounting over a telemetry tensor of per-(step, rank, stage) durations,
 * computed by CUDA kernels for sm_103a (GB300).
 *
 * Problem statement (Sec. 3, Eq. 1-2): for step t, rank r and ordered stage s
 * let d[t,r,s] >= 0 be the measured duration.  The rank-local prefix is
 * P[t,r,s] = sum_{j<=s} d[t,r,j], the frontier F[t,s] = max_r P[t,r,s] with
 * F[t,-1] = 0, the increment a[t,s] = F[t,s] - F[t,s-1] >= 0 and the exposed
 * makespan F[t,S-1] = sum_s a[t,s] (Theorem 1).  A window of steps has stage
 * share A_s = sum_t a[t,s] / sum_t F[t,S-1].
 *
 * Conventions shared by every entry point
 *   - d is int64 nanoseconds, row-major [T][R][S], contiguous, 16-byte aligned
 *     (else SF_EINVAL_ALIGN).  Stages and ranks are 0-based.
 *   - Every data pointer is a DEVICE pointer owned by the caller unless the
 *     argument says "host".  The library never allocates device memory, never
 *     frees, and never synchronizes: work is enqueued on `stream` and the call
 *     returns.  Output buffers must not alias inputs.
 *   - Host-detectable errors (shapes, null required pointers, alignment,
 *     configuration) return a negative sf_status before anything is enqueued.
 *   - Errors found on the device (invalid durations, a bounded wait that ran
 *     out) are OR-ed into the caller's device word `*status` (nullable; the
 *     caller zeroes it and reads it after its own synchronization).  When a
 *     status bit is set, the outputs of that call are unspecified.
 *   - Supported shapes: 1 <= T, 1 <= R <= 65536, 1 <= S <= 32,
 *     1 <= W <= 65536 (window length in steps), 1 <= k <= 32.
 *   - Valid durations satisfy 0 <= d < 2^47 and every rank total
 *     P[t,r,S-1] < 2^47 ns (about 39 hours per step); anything else sets
 *     SF_ST_NEGATIVE or SF_ST_RANGE.  All sums over a window then fit int64.
 *   - Ties: the lead rank of (t,s) is the LOWEST rank attaining F[t,s] (how
 *     many ranks attain it is reported by sf_frontier_ties); the leading stage
 *     of a step is the lowest stage with the largest increment.
 *   - Integer outputs are exact and deterministic (integer atomics commute);
 *     fp64 outputs are one IEEE division of two int64 values.
 */
#ifndef STAGEFRONTIER_H
#define STAGEFRONTIER_H

#include <stddef.h>
#include <stdint.h>
#include <cuda_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum sf_status {
  SF_OK = 0,
  SF_EINVAL = -1,        /* bad shape, null required pointer or bad configuration */
  SF_EINVAL_ALIGN = -2,  /* a pointer is not aligned as documented */
  SF_EUNSUPPORTED = -3,  /* shape outside the supported limits */
  SF_ECUDA = -4,         /* a CUDA runtime call (launch, attribute, driver entry) failed */
  SF_EWORKSPACE = -5     /* workspace pointer null or smaller than required */
} sf_status;

/* device status bits */
#define SF_ST_NEGATIVE 1u /* some duration (or wall time) was negative */
#define SF_ST_RANGE 2u    /* some duration, rank total or wall time was >= 2^47 */
#define SF_ST_TIMEOUT 4u  /* a bounded device-side wait gave up; outputs incomplete */
#define SF_ST_INDEX 8u    /* an index input (a rank's group id, a token, an expert) was out of range; it was skipped */
#define SF_ST_NONFINITE 16u /* training-step operators: a value that has to be finite was not */

/* Label bits (Sec. 4 Tab. core labels, App. B, App. C).  RAW_ONLY marks a
   window whose denominator is below the floor: raw advances, no shares. */
#define SF_LABEL_FRONTIER_ACCOUNTING (1u << 0)
#define SF_LABEL_DIRECT_EXPOSURE (1u << 1)
#define SF_LABEL_SYNC_WAIT_DEPENDENT (1u << 2)
#define SF_LABEL_CO_CRITICAL (1u << 3)
#define SF_LABEL_ROLE_AWARE_NEEDED (1u << 4)
#define SF_LABEL_TELEMETRY_LIMITED (1u << 5)
#define SF_LABEL_RAW_ONLY (1u << 6)

/* step_lead byte written by sf_direct_gain: low 5 bits = leading stage,
   bit 7 = the step is a confident unique leader (Sec. 4). */
#define SF_STEP_CONFIDENT 0x80u

/* Human-readable name of a status code (host string, never null). */
const char* sf_status_str(int code);

/* Number of windows a call covering global steps [t0, t0+T) touches:
   floor((t0+T-1)/W) - floor(t0/W) + 1.  Returns 0 on bad arguments. */
int64_t sf_num_windows(int64_t t0, int64_t T, int64_t W);

/* Kernels this library has launched since it was loaded (all entry points). */
uint64_t sf_launch_count(void);

/* Self-test of the device-side bounded waits every pipelined kernel uses: a
   one-CTA kernel waits on a barrier phase that never completes, gives up after
   limit_ns (0 < limit_ns <= 2 s) and ORs SF_ST_TIMEOUT into *status (device,
   required).  The kernel then exits normally; nothing faults or traps. */
sf_status sf_selftest_bounded_wait(uint64_t limit_ns, uint32_t* status, cudaStream_t stream);

/*
 * sf_frontier - Sec. 3 Eq. 1 on every step.
 *   d         [T][R][S] durations (device, 16-byte aligned).
 *   a         [T][S] increments a[t,s] (device, nullable).
 *   lead      [T][S] lowest rank attaining F[t,s] (device, nullable).
 *   makespan  [T] exposed makespan F[t,S-1] (device, nullable).
 *   status    device error word (nullable).
 * At least one output must be non-null.
 */
sf_status sf_frontier(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t* a, int32_t* lead,
                      int64_t* makespan, uint32_t* status, cudaStream_t stream);

/*
 * sf_frontier_ties - the size of the lead rank's tie set, among the
 * localization evidence of Sec. 4 (the "latest-rank tie set"; Fig. 1 has a
 * real tie at the backward boundary): ties[t,s] = #{r : P[t,r,s] = F[t,s]},
 * the number of ranks whose prefix reaches the frontier.  1 marks a unique
 * lead rank; more, a tie that sf_frontier resolved to the lowest rank.
 *   d       [T][R][S] durations (device, 16-byte aligned).
 *   a       [T][S] increments from sf_frontier on the same d (device, 8-byte
 *           aligned); F[t,s] is rebuilt as their prefix over s.
 *   ties    [T][S] int32 (device, 4-byte aligned, caller-owned).
 *   status  device error word (nullable): SF_ST_NEGATIVE / SF_ST_RANGE as in
 *           sf_frontier.
 * Reads d once more (one CTA per step range).  Errors: SF_EINVAL (null d, a
 * or ties, bad shape), SF_EINVAL_ALIGN.
 */
sf_status sf_frontier_ties(const int64_t* d, int64_t T, int64_t R, int64_t S, const int64_t* a, int32_t* ties,
                           uint32_t* status, cudaStream_t stream);

/*
 * sf_window_aggregate - Eq. 2 numerators and denominators plus per-(stage,
 * rank) credit, fused into the frontier pass.  Global step g = t0 + t belongs
 * to window floor(g / W); output row i is global window floor(t0 / W) + i,
 * i < sf_num_windows(t0, T, W).  A chunked caller passes the same buffers
 * with successive t0 and accumulate = 1 so windows that straddle chunks sum
 * correctly.
 *   X         [nW][S]    sum_t a[t,s]                            (device, required)
 *   D         [nW]       sum_t F[t,S-1]                          (device, required)
 *   E         [nW][S][R] sum of a[t,s] over steps whose lead rank is r (device, nullable)
 *   C         [nW][S][R] number of steps whose lead rank at s is r (device, nullable)
 *   step_lead [T]        leading stage argmax_s a[t,s]           (device, nullable)
 *   accumulate 0: the call first zeroes X, D, E, C; 1: adds to their contents.
 */
sf_status sf_window_aggregate(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t t0,
                              int64_t W, int64_t* X, int64_t* D, int64_t* E, int32_t* C,
                              uint8_t* step_lead, int32_t accumulate, uint32_t* status,
                              cudaStream_t stream);

/*
 * sf_window_baselines - the routing baselines the paper compares frontier
 * accounting against (Sec. 3 per-stage max and average, Props 1-2; Sec. 6
 * routing table), per window and stage, in one pass over d:
 *   M     [nW][S]    sum_t max_r d[t,r,s]                  (per-stage max)
 *   SUM   [nW][S][2] sum_t sum_r d[t,r,s] as a 128-bit (lo, hi) pair
 *                    (per-stage average times R; exact)
 *   SLOW  [nW][S]    sum_t d[t,r*,s], r* the step's slowest rank (largest total,
 *                    lowest rank on ties): the slowest-rank breakdown
 *   RANK0 [nW][S]    sum_t d[t,0,s]                          (rank-0 local total)
 * Windows, t0 and accumulate as in sf_window_aggregate; all outputs device,
 * required.
 */
sf_status sf_window_baselines(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t t0, int64_t W,
                              int64_t* M, uint64_t* SUM, int64_t* SLOW, int64_t* RANK0,
                              int32_t accumulate, uint32_t* status, cudaStream_t stream);

/*
 * sf_rank_lag - localization evidence of Sec. 4 per step and stage:
 *   L  [T][S] lag F[t,s] - median_r P[t,r,s] (lower median over ranks),
 *   dL [T][S] its increment L[t,s] - L[t,s-1] (L[t,-1] = 0),
 *   G  [T][S] max-minus-second-max gap F[t,s] - (second largest P[t,r,s]; a
 *             tie at the top counts as the second, so ties give 0; R = 1 gives 0).
 * Outputs device, nullable (at least one).  workspace: device, 256-byte
 * aligned, at least one step's scratch; sf_rank_workspace_size(T, R, S)
 * bytes (about 40 MB, so that the scratch stays in L2) processes the steps
 * in the fewest chunks that still fit L2.  The workspace is required for every
 * shape, but steps whose selection fits on chip leave it untouched; otherwise it
 * is overwritten.  It may be reused as soon as the call's work on `stream` is done.
 */
sf_status sf_rank_lag(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t* L, int64_t* dL, int64_t* G,
                      void* workspace, size_t workspace_bytes, uint32_t* status, cudaStream_t stream);

/*
 * sf_raw_spread - the raw rank spread of the Sec. 6 routing table, per window
 * and stage: sum_t (max_r d[t,r,s] - median_r d[t,r,s]), lower median over
 * ranks.  spread [nW][S] device; windows, t0 and accumulate as in
 * sf_window_aggregate; workspace as in sf_rank_lag.
 */
sf_status sf_raw_spread(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t t0, int64_t W,
                        int64_t* spread, int32_t accumulate, void* workspace, size_t workspace_bytes,
                        uint32_t* status, cudaStream_t stream);

/*
 * sf_rank_lag_windows - the same evidence as window evidence: per window and
 * stage, Lw = sum_t L[t,s] and Gw = sum_t G[t,s] (the window's delta-lag sums
 * are Lw[w][s] - Lw[w][s-1]).  Lw, Gw [nW][S] device, nullable (at least
 * one); windows, t0 and accumulate as in sf_window_aggregate; workspace as in
 * sf_rank_lag.
 */
sf_status sf_rank_lag_windows(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t t0, int64_t W,
                              int64_t* Lw, int64_t* Gw, int32_t accumulate, void* workspace, size_t workspace_bytes,
                              uint32_t* status, cudaStream_t stream);

/* Suggested workspace bytes for sf_rank_lag, sf_rank_lag_windows and sf_raw_spread (0 for a bad shape). */
size_t sf_rank_workspace_size(int64_t T, int64_t R, int64_t S);

/*
 * sf_group_aggregate - the frontier taken within role groups.  The App. A
 * contract check forbids one global frontier across ranks whose roles
 * differ (the labeler then emits role_aware_needed); with a rank -> group
 * map the frontier of Sec. 3 Eq. 1 is taken inside each group instead:
 *   F_g[t,s] = max of P[t,r,s] over the ranks r of group g (0 if g has none),
 *   a_g[t,s] = F_g[t,s] - F_g[t,s-1], F_g[t,-1] = 0,
 *   Xg [nW][G][S] sum_t a_g[t,s],  Dg [nW][G] sum_t F_g[t,S-1]   (device, required)
 * group [R] int32 device: each rank's group in [0, G); a rank whose id is
 * outside that range is left out and SF_ST_INDEX is set.  1 <= G <= 4096,
 * G*S <= 4096.  Windows, t0 and accumulate as in sf_window_aggregate.  The
 * group Xg[:, g, :], Dg[:, g] feed sf_label_gates like X, D.
 */
sf_status sf_group_aggregate(const int64_t* d, int64_t T, int64_t R, int64_t S, const int32_t* group, int64_t G,
                             int64_t t0, int64_t W, int64_t* Xg, int64_t* Dg, int32_t accumulate, uint32_t* status,
                             cudaStream_t stream);

/*
 * sf_stage_group_sum - reporting groups aggregated after the frontier
 * (Sec. 3: with gradient accumulation the ordered stage list is expanded by
 * accumulation index before the frontier, and semantic groups such as
 * "forward" or "backward" are summed only afterwards):
 *   Y [nW][K] = sum of X[w][s] over the stages s with stage_group[s] = k.
 * X [nW][S] device; stage_group [S] HOST array, values in [0, K), 1 <= K <= 32;
 * Y device, overwritten.  nW = 0 is a no-op.
 */
sf_status sf_stage_group_sum(const int64_t* X, int64_t nW, int64_t S, const int32_t* stage_group, int64_t K,
                             int64_t* Y, cudaStream_t stream);

/*
 * sf_gathered_to_steps - rank-major ingest.  The window-boundary gather of
 * Sec. 5 leaves each window's telemetry as one [R][n][S] block (each rank's
 * [n, S] buffer, in rank order).  This converts ceil(T / N) such blocks,
 * stored one after another (block b holds steps b*N .. min(T, (b+1)*N) - 1,
 * so only the last may be short), into the [T][R][S] layout every other
 * entry point reads.  src and dst device, 16-byte aligned, not overlapping.
 */
sf_status sf_gathered_to_steps(const int64_t* src, int64_t T, int64_t R, int64_t S, int64_t N, int64_t* dst,
                               cudaStream_t stream);

/*
 * sf_topk_suspects - per window, the k stages with the largest X (Sec. 4
 * routing uses the top two shares) and the k (stage, rank) pairs with the
 * largest lead-rank credit E.  Order: value descending, then lower stage,
 * then lower rank.  Entries with value 0 are not suspects; unused slots hold
 * -1 (values 0).
 *   X [nW][S], E [nW][S][R] (device; E nullable when no pair output is asked)
 *   top_stage [nW][k], top_stage_value [nW][k] (device, nullable)
 *   top_pair [nW][k][2] = (stage, rank), top_pair_value [nW][k] (device, nullable)
 */
sf_status sf_topk_suspects(const int64_t* X, const int64_t* E, int64_t nW, int64_t S, int64_t R,
                           int32_t k, int32_t* top_stage, int64_t* top_stage_value,
                           int32_t* top_pair, int64_t* top_pair_value, cudaStream_t stream);

/* Labeler thresholds as exact rationals num/den (0 <= num <= 2^31,
   0 < den <= 2^31).  Defaults (App. C): gamma_A 2/5, gamma_G 1/10,
   eta_A = eta_G 1/20, tau_C 4/5, closure_max 1/20, overlap_max 1/100,
   max_missing_ranks 0, model_fit_mask 0 (W_s = 0).  eta_Q, gamma_switch and
   gamma_elig have no published value: 1/20, 1/4, 1/2.  denom_floor_ns 1. */
typedef struct sf_ratio {
  int64_t num, den;
} sf_ratio;

typedef struct sf_label_config {
  sf_ratio gamma_A, gamma_G, eta_A, eta_G, tau_C, eta_Q, gamma_switch, gamma_elig, closure_max,
      overlap_max;
  int64_t denom_floor_ns;
  int32_t max_missing_ranks;
  uint32_t model_fit_mask; /* bit s set: workload semantics support sync-wait dependence (W_s = 1) */
} sf_label_config;

/* Fill *cfg (host) with the defaults above. */
void sf_label_config_default(sf_label_config* cfg);

/*
 * sf_window_median - the per-rank window baseline of Sec. 4 (Eq. 4): for each
 * window w (steps [wW, min((w+1)W, T)) of d, starting at d's first step), rank
 * r and stage s, the LOWER median of {d[t,r,s]}: element floor((n-1)/2) of the
 * ascending order, n the window's step count.
 *   m  [nW][R][S] (device), nW = ceil(T / W).
 */
sf_status sf_window_median(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t W,
                           int64_t* m, uint32_t* status, cudaStream_t stream);

/*
 * sf_direct_gain - the evidence pass of the labeler (Sec. 4): per window the
 * Eq. 2 numerators X and denominator D, optionally the lead-rank credit E and
 * lead counts C exactly as sf_window_aggregate defines them (so one pass over
 * d serves both), the Eq. 4 numerators
 * Y[w,s] = sum_t (F[t,S-1] - F'[t,S-1]) where F' replaces stage s by the
 * clipped baseline min(d, m) on every rank, the per-step leading stage with its
 * confidence (unique leader whose margin over the runner-up is
 * >= eta_Q * F[t,S-1], F > 0), and telemetry-quality sums (App. A).
 *   m          [nW][R][S] from sf_window_median (device).
 *   wall       [T][R] step wall times (device, nullable).
 *   other_stage index of the residual stage, or -1.
 *   X [nW][S], Y [nW][S], D [nW] (device, required; overwritten).
 *   E [nW][S][R] int64, C [nW][S][R] int32 (device, nullable; overwritten).
 *   step_lead  [T] leading stage | SF_STEP_CONFIDENT (device, required).
 *   quality    [nW][6] uint64 (device, nullable; overwritten): 128-bit sums
 *              (lo, hi) of the closure residual, the overlap error and the wall
 *              time.  With wall: residual max(0,e), overlap max(0,-e),
 *              e = wall - sum_{s != other} d.  Without wall but with
 *              other_stage: residual d[other], wall = the rank total.
 */
sf_status sf_direct_gain(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t W,
                         const int64_t* m, const int64_t* wall, int32_t other_stage,
                         sf_ratio eta_Q, int64_t* X, int64_t* Y, int64_t* D, int64_t* E, int32_t* C,
                         uint8_t* step_lead, uint64_t* quality, uint32_t* status, cudaStream_t stream);

/*
 * sf_label_gates - App. C gates per window from the evidence above: shares
 * A = X/D and gains G = Y/D (fp64), routing candidate set (shortest prefix of
 * stages by X descending reaching tau_C * D), ambiguity set E_amb = C_A u C_G
 * (stages whose X, resp. Y, is strictly within eta * D of the top), leader
 * switches between consecutive confident steps, and the label bitmask.
 *   role    [R] rank role ids (device, nullable): more than one distinct value
 *           sets ROLE_AWARE_NEEDED.
 *   missing [nW] missing-rank count per window (device, nullable).
 *   quality from sf_direct_gain (device, nullable).
 *   cfg     host pointer.
 *   labels, route_mask, amb_mask [nW] (device, required); share, gain [nW][S]
 *   (device, nullable); n_confident, n_switch [nW] int32 (device, nullable).
 */
sf_status sf_label_gates(int64_t T, int64_t R, int64_t S, int64_t W, const int64_t* X,
                         const int64_t* Y, const int64_t* D, const uint8_t* step_lead,
                         const uint64_t* quality, const int32_t* role, const int32_t* missing,
                         const sf_label_config* cfg, uint32_t* labels, uint32_t* route_mask,
                         uint32_t* amb_mask, double* share, double* gain, int32_t* n_confident,
                         int32_t* n_switch, cudaStream_t stream);

/* Workspace bytes sf_label_windows needs for (T, R, S, W); 0 on bad arguments. */
size_t sf_label_windows_workspace_size(int64_t T, int64_t R, int64_t S, int64_t W);

/*
 * sf_label_windows - the whole labeler: sf_window_median, sf_direct_gain and
 * sf_label_gates in sequence on `stream`, with intermediates (medians, X, Y,
 * D, step leaders, quality sums) in the caller's device `workspace`
 * (>= sf_label_windows_workspace_size bytes, 256-byte aligned).
 *   X, Y [nW][S], D [nW] (device, nullable): copies of the evidence.
 */
sf_status sf_label_windows(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t W,
                           const int32_t* role, const int32_t* missing, const int64_t* wall,
                           int32_t other_stage, const sf_label_config* cfg, void* workspace,
                           size_t workspace_bytes, uint32_t* labels, uint32_t* route_mask,
                           uint32_t* amb_mask, double* share, double* gain, int64_t* X,
                           int64_t* Y, int64_t* D, uint32_t* status, cudaStream_t stream);

/*
 * sf_stream_windows - the whole hot path over a tensor that lives in HOST
 * memory: the steps are cut into chunks of chunk_steps steps (a multiple of
 * W, so every chunk holds whole windows); each chunk is copied host->device on
 * `copy_stream` into one of two device staging buffers and then, on
 * `stream`, gets sf_window_median, sf_direct_gain (with lead-rank credit when
 * E/C are given), sf_topk_suspects and sf_label_gates, its windows written to
 * the output rows they belong to.  The copy of the next chunk overlaps the
 * computation of the current one when h_d is page-locked and the two streams
 * differ.  This is the chunked streaming of the largest workload
 * (Sec. 5's window-boundary delivery of rank vectors, here host to GPU).
 *   h_d        [T][R][S] host, 16-byte aligned (page-locked for overlap).
 *   staging    device, >= sf_stream_windows_staging_size(T, R, S, chunk_steps)
 *              bytes, 16-byte aligned: two chunk buffers.
 *   workspace  device, >= sf_label_windows_workspace_size(min(chunk_steps, T),
 *              R, S, W) bytes: one chunk's medians and step leaders.
 *   outputs (device) indexed by global window: X, Y [nW][S], D [nW] required;
 *   E [nW][S][R], C [nW][S][R], top_stage, top_pair [nW][k][2],
 *   top_pair_value [nW][k], share, gain [nW][S] nullable; labels, route_mask,
 *   amb_mask [nW] required.  No telemetry-quality or role inputs.
 * The call creates and releases four CUDA events; it allocates no memory.
 * Returns when everything is enqueued.
 */
sf_status sf_stream_windows(const int64_t* h_d, int64_t T, int64_t R, int64_t S, int64_t W, int32_t k,
                            int64_t chunk_steps, const sf_label_config* cfg, int64_t* staging,
                            size_t staging_bytes, void* workspace, size_t workspace_bytes, int64_t* X,
                            int64_t* Y, int64_t* D, int64_t* E, int32_t* C, int32_t* top_stage,
                            int32_t* top_pair, int64_t* top_pair_value, uint32_t* labels,
                            uint32_t* route_mask, uint32_t* amb_mask, double* share, double* gain,
                            uint32_t* status, cudaStream_t stream, cudaStream_t copy_stream);

/* Device staging bytes sf_stream_windows needs; 0 on bad arguments. */
size_t sf_stream_windows_staging_size(int64_t T, int64_t R, int64_t S, int64_t chunk_steps);

/*
 * sf_stream_gathered_windows - sf_stream_windows over telemetry as the
 * window-boundary gather delivers it (Sec. 5): h_g holds the windows'
 * [R][n][S] blocks one after another (window w's block at element w*W*R*S,
 * the last window possibly short), in host memory.  Each chunk is copied as
 * is, converted on the device (sf_gathered_to_steps) into a third staging
 * buffer, and then takes the same path.  Arguments and outputs as in
 * sf_stream_windows; staging >= sf_stream_gathered_staging_size(...) bytes.
 */
sf_status sf_stream_gathered_windows(const int64_t* h_g, int64_t T, int64_t R, int64_t S, int64_t W, int32_t k,
                                     int64_t chunk_steps, const sf_label_config* cfg, int64_t* staging,
                                     size_t staging_bytes, void* workspace, size_t workspace_bytes, int64_t* X,
                                     int64_t* Y, int64_t* D, int64_t* E, int32_t* C, int32_t* top_stage,
                                     int32_t* top_pair, int64_t* top_pair_value, uint32_t* labels,
                                     uint32_t* route_mask, uint32_t* amb_mask, double* share, double* gain,
                                     uint32_t* status, cudaStream_t stream, cudaStream_t copy_stream);
size_t sf_stream_gathered_staging_size(int64_t T, int64_t R, int64_t S, int64_t chunk_steps);

/*
 * sf_label_windows_noalloc - sf_label_windows for callers that cannot
 * allocate device memory.  The paper has no counterpart; this is a
 * deployment variant of the labeler above.  It exists because an always-on
 * monitor runs inside someone else's training job: the framework's caching
 * allocator owns the device memory there, and a cudaMalloc issued from the
 * monitoring hook can block on or synchronize the device (stalling the very
 * step it measures) and carve memory out of that pool; a side-car with a
 * fixed memory budget may have no allocator to call at all.
 *
 * Scratch: one static device array of SF_STATIC_SCRATCH_BYTES (16 MiB) in
 * this library, held by every GPU that loads the library until the process
 * exits.  A problem whose sf_label_windows_workspace_size exceeds it returns
 * SF_EWORKSPACE before anything is enqueued.  The call allocates nothing and
 * frees nothing.
 *
 * Set-up: the first call on each device looks up the array's device address
 * (cudaGetSymbolAddress) with that device current, and caches it; make that
 * first call before any stream capture.  The cached address belongs to the
 * device's current primary context: after cudaDeviceReset (or any other
 * reset of that context) the module is loaded afresh and the array may move,
 * so do not call this entry point again in a process that has reset the
 * device.
 *
 * Sharing: all calls on a device use the same array, and it keeps whatever
 * the last call left there.  Each call zeroes the parts it accumulates into,
 * so calls ordered on one stream are independent; calls that can overlap on
 * the GPU (other streams without an ordering event, concurrent host threads)
 * race on the array and corrupt each other's results.
 *
 * Arguments, outputs and errors are those of sf_label_windows, without the
 * workspace pair.
 */
#define SF_STATIC_SCRATCH_BYTES (16u * 1024u * 1024u)

sf_status sf_label_windows_noalloc(const int64_t* d, int64_t T, int64_t R, int64_t S, int64_t W,
                                   const int32_t* role, const int32_t* missing, const int64_t* wall,
                                   int32_t other_stage, const sf_label_config* cfg, uint32_t* labels,
                                   uint32_t* route_mask, uint32_t* amb_mask, double* share,
                                   double* gain, int64_t* X, int64_t* Y, int64_t* D,
                                   uint32_t* status, cudaStream_t stream);

/*
 * Training-step operators.  The monitor runs inside the job whose stages it
 * times; these entry points compute, in that job's own step, what a report
 * sets beside a stage's exposed time: the experts' loads (why one rank's
 * forward stage leads the frontier), the loss with its clip share and KL
 * term, and the gradient norm with the clipping that follows it.  The general
 * conventions above hold (caller's device memory and stream, no allocation,
 * no synchronization, host errors before anything is enqueued), except:
 *   - Empty calls are valid: N = 0 rows, T = 0 tokens, n = 0 tensors.
 *   - Data may start at any element's alignment; 16-byte aligned rows are
 *     read and written faster.
 *   - The outputs are defined when SF_ST_INDEX or SF_ST_NONFINITE is set: each
 *     entry point says what was left out.
 *   - Sums are held in 32 bits or more and added in a fixed order: the same
 *     call on the same device gives the same bits.
 */
typedef enum sf_dtype { SF_F32 = 0, SF_BF16 = 1, SF_F16 = 2 } sf_dtype;

typedef struct sf_policy_config {
  float clip_low, clip_high; /* the ratio's bounds are 1 - clip_low and 1 + clip_high; 0 <= clip_low <= 1 */
  float kl_coef;             /* beta >= 0 */
  float inv_temperature;     /* tau, 0 < tau <= 1e6: the policy is softmax(tau * logits) */
} sf_policy_config;

#define SF_POLICY_DIRECT_ROWS 1024

/*
 * sf_policy_loss - the clipped policy loss with a KL term, from the logits,
 * and its gradient.  For row (token) n with logits z, chosen token y, weight
 * w != 0 and upstream gradient g:
 *   lp   = tau z_y - log sum_j exp(tau z_j)
 *   r    = exp(lp - old),  held = clamp(r, 1 - clip_low, 1 + clip_high)
 *   pg   = -min(r A, held A);  the row is clipped if held A < r A
 *   kl   = exp(ref - lp) - (ref - lp) - 1       (0 without ref_logp)
 *   loss = pg + beta kl
 *   dz_j = g w tau c ([j = y] - exp(tau z_j - log sum)),
 *          c = (clipped ? 0 : -r A) + beta (1 - exp(ref - lp))
 * A row of weight 0 is not read: its log-probability, loss and gradient are 0.
 * A logit of -inf is a token that is ruled out: probability and gradient 0.
 *   logits    [N] rows of V, `ld` elements apart (ld >= V), of type dtype
 *   target    [N] int64, the chosen tokens
 *   old_logp, advantage [N] f32;  ref_logp [N] f32 (nullable: no KL term)
 *   weight    [N] f32 (nullable: 1/N each)
 *   grad_out  f32 (device, nullable: 1), the upstream gradient g of the loss
 *   logp      [N] f32 (nullable), lp;  token_loss [N] f32 (nullable), loss
 *   stats     [4] f32: the sums over rows of w times loss, pg, kl, clipped; a sum
 *             beyond the largest f32 is infinite
 *   dlogits   [N] rows of V, ldd elements apart, of type dtype (nullable: no
 *             gradient); may be `logits` itself with ldd = ld, else the two
 *             must not overlap.  Rounded once, to nearest even.
 *   workspace device, 16-byte aligned, sf_policy_loss_workspace_size(N, V) bytes;
 *             may be null for up to SF_POLICY_DIRECT_ROWS rows with logp given
 * A row whose token is not in [0, V) is left out like one of weight 0, with
 * SF_ST_INDEX; so is one whose loss, KL term, weight or derivative is not
 * finite (a NaN or +inf logit, no logit above -inf), with SF_ST_NONFINITE.
 * N < 2^31, 1 <= V <= 2^30.
 */
sf_status sf_policy_loss(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld, const int64_t* target,
                         const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                         const sf_policy_config* cfg, const float* grad_out, float* logp, float* token_loss,
                         float* stats, void* dlogits, int64_t ldd, void* workspace, size_t workspace_bytes,
                         uint32_t* status, cudaStream_t stream);

/* Workspace bytes of sf_policy_loss; 0 on bad arguments and for N = 0. */
size_t sf_policy_loss_workspace_size(int64_t N, int64_t V);

#define SF_SCORE_SOFTMAX 0
#define SF_SCORE_SIGMOID 1

typedef struct sf_route_config {
  int32_t k;          /* experts a token is sent to, 1 <= k <= 32 */
  int32_t score;      /* SF_SCORE_SOFTMAX or SF_SCORE_SIGMOID */
  int32_t groups;     /* the E experts are `groups` runs of E / groups, 1 <= groups <= 32 */
  int32_t top_groups; /* groups a token may use, k <= top_groups * E / groups */
  int32_t group_top;  /* a group's value is the sum of its 1 or 2 largest choice values */
  int32_t renorm;     /* 1: the weights of a token's experts sum to `scale` */
  float scale;        /* finite */
} sf_route_config;

/*
 * sf_route_experts - the router of a layer of experts.  For token t with
 * logits z over E experts:
 *   choice value  u_e = z_e + bias_e (softmax) or 1 / (1 + exp(-z_e)) + bias_e
 *                 (sigmoid): the bias balances the loads and enters nothing else
 *   group value   the sum of the group_top largest u in the group
 *   chosen        the k largest u among the experts of the top_groups groups of
 *                 largest value; equal values go to the lower group or expert
 *   weight        softmax: scale exp(z_e) / sum exp(z_j), j over the chosen
 *                 (renorm) or over all experts; sigmoid: scale s_e / sum s_j over
 *                 the chosen (renorm; 0 where that sum is 0) or scale s_e
 * u is computed in 32 bits exactly as written, each operation rounded to
 * nearest.  An expert whose logit or bias is -inf is not available: it is
 * never chosen and a group without any has no value.  Where fewer than k
 * experts are available the last slots hold index -1, weight 0 and count for
 * no expert.  An expert whose choice value is NaN, or +inf logit under softmax,
 * is taken as not available, with SF_ST_NONFINITE.
 *   logits [T] rows of E, ld elements apart;  bias [E] f32 (nullable: 0)
 *   index  [T][k] int32, weight [T][k] f32, by falling choice value
 *   load   [E] int32 (nullable): tokens sent to each expert; accumulate 1 adds
 *          to its contents (the micro-batches of a step), 0 overwrites them
 * T < 2^31, 1 <= E <= 1024.
 */
sf_status sf_route_experts(const void* logits, int32_t dtype, int64_t T, int64_t E, int64_t ld, const float* bias,
                           const sf_route_config* cfg, int32_t* index, float* weight, int32_t* load,
                           int32_t accumulate, uint32_t* status, cudaStream_t stream);

/*
 * sf_route_experts_grad - the gradient of the router's logits from that of the
 * weights; the choice itself and the bias have none.  With S the sum that
 * `weight` above divides by, s the scores, q_e = exp(z_e) / S, dw the upstream
 * gradient and j over the chosen:
 *   sigmoid  renorm   dz_e = scale s_e (1 - s_e) / S (dw_e - sum_j dw_j s_j / S)
 *            else     dz_e = scale s_e (1 - s_e) dw_e
 *   softmax           dz_e = scale q_e (dw_e [e chosen] - sum_j q_j dw_j)
 * and 0 for experts that are not chosen, but for softmax without renorm.
 *   index   [T][k] as sf_route_experts wrote it (distinct within a token)
 *   dweight [T][k] f32;  dlogits [T] rows of E, ldd elements apart, of type
 *   dtype, rounded once; must not overlap logits
 * cfg's groups, top_groups and group_top are not used.  A slot whose index is
 * -1 is empty; any other index outside [0, E) is skipped with SF_ST_INDEX.
 * Where S is 0, or (softmax) not finite, the row's gradient is 0; the latter
 * sets SF_ST_NONFINITE.
 */
sf_status sf_route_experts_grad(const void* logits, int32_t dtype, int64_t T, int64_t E, int64_t ld,
                                const int32_t* index, const float* dweight, const sf_route_config* cfg,
                                void* dlogits, int64_t ldd, uint32_t* status, cudaStream_t stream);

/*
 * sf_grad_norm - the 2-norm over n gradient tensors and of each of them.
 *   data, numel, dtype  HOST arrays of n: each tensor's device pointer (aligned
 *               to its element; unused where numel is 0), element count and
 *               sf_dtype.  Read before the call returns.
 *   norm        [1] f32: sqrt(sum of squares over all tensors)
 *   tensor_norm [n] f32 (nullable): each tensor's own
 *   workspace   device, 16-byte aligned, sf_grad_workspace_size(n) bytes; may be
 *               null where sf_grad_needs_workspace says 0
 * Squares that leave the range of 32 bits are summed in 64.  Where the norm is
 * not finite (or above the largest f32) SF_ST_NONFINITE is set and `norm`
 * holds what it is; tensor_norm tells which tensors are the cause.
 * n <= 2^20, each numel < 2^40.
 */
sf_status sf_grad_norm(const void* const* data, const int64_t* numel, const int32_t* dtype, int64_t n, float* norm,
                       float* tensor_norm, void* workspace, size_t workspace_bytes, uint32_t* status,
                       cudaStream_t stream);

/*
 * sf_grad_clip - sf_grad_norm, then every gradient times
 *   coef = min(1, max_norm / (norm + eps)),
 * rounded once.  out: HOST array of n device pointers, each tensor's result
 * (same type and count, not overlapping any input other than its own), or
 * null: in place, where nothing is written for coef = 1.  Where the norm is not finite
 * coef is NaN and the gradients are passed on unscaled, so that the caller can
 * skip the step.  max_norm > 0, eps >= 0; coef [1] f32 (device, nullable).
 */
sf_status sf_grad_clip(const void* const* data, void* const* out, const int64_t* numel, const int32_t* dtype,
                       int64_t n, float max_norm, float eps, float* norm, float* coef, float* tensor_norm,
                       void* workspace, size_t workspace_bytes, uint32_t* status, cudaStream_t stream);

/* Workspace bytes sf_grad_norm and sf_grad_clip need for n tensors on the
   current device; 0 on bad arguments. */
size_t sf_grad_workspace_size(int64_t n);

/* Whether sf_grad_norm and sf_grad_clip need a workspace for these tensors
   (HOST arrays): 0 for up to 960 tensors of up to 393216 packs of 16 bytes (6 MB,
   the last pack of each tensor counted whole), which take one launch and use no
   workspace, and on bad arguments. */
int32_t sf_grad_needs_workspace(const int64_t* numel, const int32_t* dtype, int64_t n);

/*
 * The operators around a policy's layers: what its tokens pass between the
 * router and the loss (the gated feed-forward product, dropout on the residual
 * stream), and where the tokens that sf_policy_loss scores come from (drafted
 * tokens verified against the policy).  The conventions of the training-step
 * operators hold.
 */
#define SF_ACT_SILU 0      /* g / (1 + exp(-g)) */
#define SF_ACT_GELU 1      /* g (1 + erf(g / sqrt 2)) / 2 */
#define SF_ACT_GELU_TANH 2 /* g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2 */
#define SF_ACT_RELU 3      /* max(g, 0), slope 0 at 0 */

/*
 * sf_gated_ffn - the gated feed-forward product: both projections, the
 * activation and the product in one pass,
 *   h = act(x Wg^T) * (x Wu^T)
 *   x       [T] rows of H, ldx elements apart, of type dtype
 *   w_gate, w_up [F] rows of H, ldw elements apart, of type dtype
 *   h       [T] rows of F, ldh elements apart, of type dtype; must not overlap an input
 *   workspace device, 16-byte aligned, sf_gated_ffn_workspace_size(...) bytes;
 *             may be null where that is 0
 * Products are summed in f32 and h is rounded once.  bf16 and f16 go by the
 * tensor cores; rows of x or weights that do not all start on 16 bytes are
 * copied to the workspace first.  The tensor cores cut their sums off instead of
 * rounding them: a sum of 4096 products of one sign is low by up to 1.4e-5 of it, of
 * 8192 by 3.5e-5, where a rounding to bf16 or f16 is up to 3.9e-3 or 4.9e-4.  f32 goes by
 * the tensor cores too, each value as the sum of three bf16 (exact for values of
 * 2^-109 and more; what is below 2^-134 is lost), in runs of 256 products that are
 * added in f32: with the error of f32 sums.  NaN and infinities go where the formula
 * takes them, but for f32 with more than a few tokens, where an infinity may also
 * make NaN.  T, H, F < 2^31, and T H, T F, F H < 2^40.
 */
sf_status sf_gated_ffn(const void* x, int32_t dtype, int64_t T, int64_t H, int64_t ldx, const void* w_gate,
                       const void* w_up, int64_t F, int64_t ldw, int32_t act, void* h, int64_t ldh, void* workspace,
                       size_t workspace_bytes, uint32_t* status, cudaStream_t stream);

/*
 * sf_gated_ffn_grad - its gradient from dh; both projections are computed
 * again, so that nothing of the size of h is kept between the passes:
 *   g = x Wg^T, u = x Wu^T, dg = dh u act'(g), du = dh act(g)
 *   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x
 *   dh      [T] rows of F, lddh elements apart, of type dtype
 *   dx      [T] rows of H, lddx elements apart, of type dtype (nullable)
 *   dw_gate, dw_up [F] rows of H, lddw elements apart, of type dw_dtype, which is
 *           dtype or SF_F32 (nullable, both or none)
 *   h       [T] rows of F, ldh elements apart: the product itself once more, for
 *           the projection behind it (nullable)
 *   accumulate 1: the weights' gradients are added to their contents (the
 *           micro-batches of a step), 0: they overwrite them
 *   workspace device, 16-byte aligned, sf_gated_ffn_workspace_size(...) bytes
 * At least one of dx, the weights' gradients and h.  dg and du are rounded once
 * to dtype between the products, as the tensor cores take them (f32: not rounded): in
 * f16 they are infinite above 65504 and 0 below 2^-25, also for weights' gradients in
 * f32.  These are summed in runs of 256 tokens that are added in f32.  Outputs must
 * not overlap inputs or one another.  Without tokens (T = 0) the weights'
 * gradients are 0, or stay as they are with accumulate.
 */
sf_status sf_gated_ffn_grad(const void* x, int32_t dtype, int64_t T, int64_t H, int64_t ldx, const void* w_gate,
                            const void* w_up, int64_t F, int64_t ldw, int32_t act, const void* dh, int64_t lddh,
                            void* dx, int64_t lddx, void* dw_gate, void* dw_up, int32_t dw_dtype, int64_t lddw,
                            int32_t accumulate, void* h, int64_t ldh, void* workspace, size_t workspace_bytes,
                            uint32_t* status, cudaStream_t stream);

/* Workspace bytes of sf_gated_ffn (grad = 0) and sf_gated_ffn_grad (grad = 1) on the current device.
   aligned: 1 if x, w_gate and w_up start on 16 bytes and ldx, ldw are multiples
   of 16 bytes.  0 on bad arguments and for T = 0. */
size_t sf_gated_ffn_workspace_size(int32_t dtype, int64_t T, int64_t H, int64_t F, int32_t aligned, int32_t grad);

/*
 * sf_dropout - out = residual + m x, m = 0 with probability p, else 1 / (1 - p),
 * with a mask from counters that is never stored.  Element (n, j) is kept if
 *   b >= t,  t = floor(65536 p + 1/2),
 * with b the 16-bit number j mod 8 (low half of each word first) of the four
 * words that Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC11) gives for the
 * counter (floor(j / 8), n, offset mod 2^32, floor(offset / 2^32)) under the key
 * (seed mod 2^32, floor(seed / 2^32)), and is then multiplied by 65536 / (65536 - t).
 * The gradient of x is this call on out's gradient with the same key and
 * without residual; the residual's is out's own.
 *   x        [N] rows of D, ldx elements apart, of type dtype
 *   key      [2] uint64, device: seed and offset, read when the kernel runs (a
 *            replayed graph draws anew once the caller has moved the offset)
 *   residual [N] rows of D, ldr elements apart, of type dtype (nullable)
 *   out      [N] rows of D, ldo elements apart, of type dtype, rounded once; may
 *            be x or residual itself (with its spacing), else must not overlap them
 * A dropped element is not read into the sum: its NaN or infinity does not
 * matter.  0 <= p <= 1; N, D < 2^31.
 */
sf_status sf_dropout(const void* x, int32_t dtype, int64_t N, int64_t D, int64_t ldx, float p, const uint64_t* key,
                     const void* residual, int64_t ldr, void* out, int64_t ldo, cudaStream_t stream);

#define SF_VERIFY_MAX_DRAFT 64

/*
 * sf_verify_draft - drafted tokens against the policy's rows, by given random
 * numbers: what is kept is distributed as the policy's own samples are.  For
 * sequence b with n drafted tokens y_i, p_i = softmax(tau target_i) and
 * q_i = softmax(tau draft_i):
 *   y_i is accepted while  uniform_i q_i(y_i) < p_i(y_i);  k is the first that is not
 *   next token  the j of largest r_j / noise_j (equal values: the lowest), with
 *               r = max(p_k - q_k, 0) if k < n (p_k if no r_j is above 0), r = p_n if k = n
 * where noise holds draws of the exponential distribution of mean 1.  Without
 * draft (tokens that were looked up) q_i is 1 at y_i.  Greedy (neither uniform
 * nor noise): y_i is accepted while it is the first of the largest logits, which
 * is also the next token.  n = 0 samples a token from each row.
 *   target  [B (L + 1)] rows of V, ldt elements apart, of type dtype: row b (L + 1) + i
 *           is the policy's before token i of sequence b
 *   draft   [B L] rows of V, ldq elements apart, of type dtype (nullable)
 *   token   [B][L] int64;  length [B] int32 (nullable: L each), drafted tokens of each sequence
 *   uniform [B][L] f32 in [0, 1);  noise [B][V] f32 above 0; both or neither
 *   out_token [B][L + 1] int64: the accepted tokens, the next one, then -1
 *   accepted  [B] int32: k
 *   logp    [B][L + 1] f32 (nullable): log p of the tokens of out_token, 0 behind
 *           them: the old_logp of sf_policy_loss
 * Probabilities are held in 32 bits.  Rows behind a sequence's length are not
 * read, and those behind the one where it stops need not be.  A token outside [0, V) is not accepted and the next one is drawn from p
 * in its place, a length outside [0, L] is taken as the nearest one, both with
 * SF_ST_INDEX.  Where a row that is needed has a NaN or +inf logit or none above
 * -inf, or no entry can be drawn (its noise is not above 0), the sequence ends
 * with next token -1, log-probability 0 and SF_ST_NONFINITE.
 * B (L + 1) < 2^31, 0 <= L <= SF_VERIFY_MAX_DRAFT, 1 <= V <= 2^24, 0 < tau <= 1e6.
 */
sf_status sf_verify_draft(const void* target, int32_t dtype, int64_t B, int64_t L, int64_t V, int64_t ldt,
                          const void* draft, int64_t ldq, const int64_t* token, const int32_t* length,
                          const float* uniform, const float* noise, float inv_temperature, int64_t* out_token,
                          int32_t* accepted, float* logp, uint32_t* status, cudaStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* STAGEFRONTIER_H */
