/*
 * ftkmeans.h -- C boundary of the MI355X (gfx950) K-means hot path.
 *
 * One Lloyd iteration of K-means (paper Section 2) is
 *     assignment  label_i = argmin_j || X_i - C_j ||_2                       (Eq. 1)
 *     update      C_j     = mean of the points with label j                  (Eq. 2)
 * The assignment is evaluated through the expansion of Section 3.1.2,
 *     || x - c ||^2 = sum_d x_d^2 + sum_d c_d^2 - 2 sum_d x_d c_d,
 * whose last term is a dense [N x D] by [D x K] contraction on the matrix cores with the
 * per-point argmin fused into its epilogue (Sections 3.1.3-3.1.5), optionally protected by
 * the online checksum scheme of Sections 2.3 and 4 (detect, locate, correct one corrupted
 * accumulator element per checked tile before the argmin reads it).
 *
 * Conventions common to every call
 *   - N points, D features, K clusters.  X is [N x D], C is [K x D], both row-major and
 *     contiguous, element type given by `dtype`.
 *   - Every array pointer is a DEVICE pointer owned by the caller unless marked (host).
 *     The library allocates no device memory: scratch comes from `workspace`, which must
 *     hold at least ftk_workspace_bytes(...) bytes and be 256-byte aligned.  Workspace
 *     contents need not survive between calls.
 *   - Calls only enqueue work on `hip_stream` (a hipStream_t; NULL = the default stream)
 *     and return without waiting, except where stated.  Calls that share a workspace must be
 *     ordered on one stream.
 *   - Distances are SQUARED Euclidean distances (the square root is dropped, Section 3.1.2).
 *   - Exact ties go to the lowest centroid index.  An empty cluster keeps its centroid.
 *   - Errors are reported by return code, never by abort; ftk_last_error() gives the text of
 *     the last failure on the calling thread.  Argument, alignment and workspace errors are
 *     found before anything is enqueued; a HIP runtime failure (FTK_EDEVICE) may leave kernels of
 *     the failed call on the stream, and the outputs are then undefined.
 */
#ifndef FTKMEANS_H
#define FTKMEANS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FTK_OK = 0,
    FTK_EINVAL = 1,        /* bad shape, NULL pointer, unknown enum value            */
    FTK_EALIGN = 2,        /* a pointer is not aligned to its element size / 256 B   */
    FTK_EWORKSPACE = 3,    /* workspace missing or too small                         */
    FTK_EDEVICE = 4,       /* a HIP runtime call failed or the device is not gfx950  */
    FTK_EUNCORRECTABLE = 5 /* reserved: never returned; see ftk_ft_stats.uncorrectable   */
} ftk_status;

/* FTK_BF16 and FTK_F16 are taken by the ftk_route_*, ftk_mx4_*, ftk_xent* and ftk_adamw_* calls alone. */
typedef enum { FTK_F32 = 0, FTK_F64 = 1, FTK_BF16 = 2, FTK_F16 = 3 } ftk_dtype;

/* Fault-tolerance mode of the contraction (Section 4).
 *   OFF     : no checksums.
 *   DETECT  : checksums carried and verified, mismatches only counted.
 *   CORRECT : a mismatching tile is repaired in place from its location-encoded checksums
 *             (Section 4.1); if the location cannot be decoded the tile is recomputed.
 *             As in the paper, an error smaller than the detection threshold (the rounding
 *             noise of the checksum comparison) passes unnoticed; it can change the label
 *             of a point only if that point's two best scores are closer than the threshold.
 *   STRICT  : CORRECT, and in addition every point whose decision an error below the threshold
 *             could have changed - its best scores are closer than the largest checksum
 *             residual seen for that point plus half the threshold for rounding noise - is
 *             settled by exact re-evaluation, so the labels equal those of a fault-free run
 *             whatever single error occurred per checked tile.  Costs the exact re-evaluation
 *             of those points.  This is the mode the benchmark reports overhead for. */
typedef enum { FTK_FT_OFF = 0, FTK_FT_DETECT = 1, FTK_FT_CORRECT = 2, FTK_FT_STRICT = 3 } ftk_ft_mode;

/* One injected soft error (fault model of Section 2.1): flip `bit` of accumulator register
 * `reg` of lane `lane`, in the `tile`-th output tile that wave `wave` of workgroup
 * `workgroup` finishes, right after its matrix instructions and before verification.
 * Fields other than `workgroup` are reduced modulo the extents ftk_assign_geometry reports,
 * so every descriptor is valid; a workgroup index beyond the grid never fires. */
typedef struct {
    uint32_t workgroup, wave, tile, reg, lane, bit;
} ftk_fault;

/* Counters accumulated (atomically added to) by ftk_kmeans_assign; zero them beforehand. */
typedef struct {
    uint64_t tiles_checked;  /* per-lane-group checksum comparisons made                  */
    uint64_t injected;       /* fault descriptors that fired                              */
    uint64_t detected;       /* checksum mismatches above the threshold                   */
    uint64_t corrected;      /* repaired from the decoded location                        */
    uint64_t recomputed;     /* location not decodable -> tile recomputed                 */
    uint64_t uncorrectable;  /* update step only: a recomputed pass mismatched again; the
                                assignment recomputes outside the matrix path and never
                                produces it                                               */
    uint64_t refined;        /* points whose best scores were closer than the rounding-
                                error bound and were re-evaluated exactly by the refine
                                kernel (none in small unprotected calls, which evaluate
                                every distance exactly)                                   */
    uint64_t max_residual_ppm; /* largest fault-free checksum residual seen, in millionths
                                of the detection threshold (maximised, not added)        */
} ftk_ft_stats;

/* Launch geometry of the assignment kernel for a problem, for building fault lists. */
typedef struct {
    uint32_t workgroups, waves_per_workgroup, tiles_per_wave, regs_per_tile, lanes, bits;
} ftk_geometry;

/* Bytes of workspace sufficient for any of the three calls below on this problem.  FTK_FT_OFF asks for
 * more than the protected modes, for buffers of faster paths that only unprotected calls take; such a
 * call also accepts a workspace of a protected mode's size, and then runs without them (mindist may
 * differ in the last places). */
size_t ftk_workspace_bytes(ftk_dtype dtype, int64_t N, int32_t D, int32_t K, ftk_ft_mode ft);

ftk_status ftk_assign_geometry(ftk_dtype dtype, int64_t N, int32_t D, int32_t K, ftk_ft_mode ft,
                               ftk_geometry *out /* (host) */);

/* (host) The two error scales of the assignment kernel chosen for a problem (16-byte aligned X
 * and C assumed), both as multiples of B_i = ||x_i|| max_j||c_j|| + max_j||c_j||^2 / 2, in units
 * of the score s_ij = x_i.c_j - ||c_j||^2/2 (half a squared distance):
 *   detect_coef : checksum detection threshold of Section 2.3 / 4.1 ("a defined threshold"): a
 *                 corrupted score is noticed when the error exceeds detect_coef * B_i; 0 with
 *                 fault tolerance off.  In FTK_FT_CORRECT a smaller error passes and can move
 *                 point i only between centroids whose squared distances differ by less than
 *                 2 * detect_coef * B_i; in FTK_FT_STRICT it cannot move it at all.
 *   band_coef   : scores closer than band_coef * B_i are not ordered by the matrix path but
 *                 settled by exact re-evaluation.
 * Both describe the fp32 / fp64 matrix kernel of the problem, which is what runs with checksums or
 * listed faults; an unprotected call may take the scan instead, which settles a wider band of its
 * own and leaves no error of this form in its distances. */
ftk_status ftk_ft_thresholds(ftk_dtype dtype, int64_t N, int32_t D, int32_t K, ftk_ft_mode ft,
                             double *detect_coef /* (host) */, double *band_coef /* (host) */);

/* (host) Consistency probe of the workspace layout: the kernels pad the K centroid rows up to
 * whole chunks of their own blocking (Section 3.2: several tile shapes per problem), and the
 * prologue writes -||c||^2/2 for every padded row.  Reports the largest padded row count over
 * every kernel variant and fault-tolerance mode that can be dispatched or forced for the problem,
 * and the rows the workspace reserves; planned_max <= reserved must hold.  The scan of unprotected
 * calls pads and reserves by itself: where it falls short, its figures are reported instead. */
ftk_status ftk_plan_padded_rows(ftk_dtype dtype, int64_t N, int32_t D, int32_t K,
                                int64_t *planned_max /* (host) */, int64_t *reserved /* (host) */);

/* Assignment step, Eq. (1), Sections 3.1.2-3.1.5 and 4.
 *   X [N x D], C [K x D]  in  : read only.
 *   labels [N] int32      out : index of the nearest centroid.
 *   mindist [N] (dtype)   out : squared distance to it, >= 0; may be NULL.  Accuracy: points whose
 *                               decision was settled by exact re-evaluation, every point of the
 *                               scan that unprotected calls with enough centroids take (bf16
 *                               matrix instructions on split operands, or fp16 ones on rounded
 *                               operands, name the centroid, the distance is evaluated from the
 *                               rows: in dtype, where the point was settled in double and rounded;
 *                               for all points in double where a problem is large enough for fp16
 *                               operands, whichever of the two forms runs), every point of the
 *                               one-launch kernels that small unprotected calls take (in double,
 *                               rounded once), and every point of the register-resident fp32
 *                               kernels (D <= 32; 32 < D <= 128 where that kernel is
 *                               dispatched), get the direct-difference value
 *                               (relative error of a few units in the last place of the
 *                               distance).  Otherwise the value comes from the expanded form of
 *                               Section 3.1.2, whose cancellation leaves an ABSOLUTE error of up
 *                               to 1.5 * band_coef * (||x_i|| max||c|| + max||c||^2/2) with
 *                               band_coef from ftk_ft_thresholds - small against the distance
 *                               unless the data sit far from the origin.
 *   faults [n_faults]     in  : soft errors to inject; NULL / 0 for none.  Ignored when
 *                               ft == FTK_FT_OFF is combined with n_faults == 0 only; with
 *                               FT off, listed faults are still injected (and corrupt the
 *                               result) so that the unprotected baseline can be observed.
 *   stats                 i/o : counters, may be NULL.
 * Requires 1 <= N, 1 <= D, 1 <= K, N*D < 2^40. */
ftk_status ftk_kmeans_assign(ftk_dtype dtype, const void *X, const void *C, int64_t N, int32_t D,
                             int32_t K, int32_t *labels, void *mindist, ftk_ft_mode ft,
                             const ftk_fault *faults, int32_t n_faults, ftk_ft_stats *stats,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/* ftk_kmeans_assign for callers that cannot allocate device memory or size a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * kernels and results as ftk_kmeans_assign, but the scratch (half norms, checksum rows, the
 * refine work-list and its counters) lives in a static device array inside the library:
 * ftk_static_scratch_bytes() = 16 MiB per GPU the library runs on, held until the process ends.
 * The call allocates nothing (no hipMalloc / hipFree, no events; the profiling aid below does
 * not apply to it).  A problem whose scratch exceeds the array (roughly N > 4 million points, or
 * K*D beyond a few million) is rejected with FTK_EWORKSPACE and nothing is enqueued; one that fits
 * only without the buffers of the scan (16 bytes per point and more) runs on the fp32 / fp64 matrix
 * kernels, whose distances may differ in the last places.  Every call
 * on a GPU shares that GPU's array: calls must be ordered on one stream; calls that overlap on
 * one GPU race.  The buffer keeps the last call's contents; everything that must start at zero
 * is cleared by the call itself. */
size_t ftk_static_scratch_bytes(void);
ftk_status ftk_kmeans_assign_static(ftk_dtype dtype, const void *X, const void *C, int64_t N, int32_t D,
                                    int32_t K, int32_t *labels, void *mindist /* nullable */,
                                    ftk_ft_mode ft, const ftk_fault *faults, int32_t n_faults,
                                    ftk_ft_stats *stats /* nullable */, void *hip_stream);

/* Assignment step on the reduced-precision matrix path - the counterpart of the paper's TF32
 * tensor-core variant (Section 3.1.5; gfx950 has no TF32 format, its fast matrix format is bf16).
 * Same outputs and tie rule as ftk_kmeans_assign with fault tolerance off.  fp32 operands are
 * split into bf16 pieces and the piece products are accumulated in fp32 by the bf16 matrix
 * instructions: three pieces each and the six largest products for D <= 32, two pieces each and
 * all four products for 32 < D <= 128 (the wider rows' instruction count makes the certified
 * bound of the three-piece form nearly as wide, see ftk_fast_plan's band_coef).  The error bound
 * of that evaluation is known, and points whose best scores fall inside it are settled by exact
 * re-evaluation as in the fp32 path, so labels meet the same tolerance (identical to the exact
 * arg-min except on near-exact ties) and mindist is the exact-form distance to the chosen
 * centroid.
 * Covers dtype == FTK_F32 with D <= 128 and D a multiple of 4, X and C 16-byte aligned; anything
 * else returns FTK_EINVAL / FTK_EALIGN.
 * ft, faults, stats as for ftk_kmeans_assign: the paper protects its tensor-core variant with the
 * same checksums as the fp32 one (Sections 3.1.5 and 4), and so does this path - tiles of 30
 * centroids whose two checksum rows are split into bf16 pieces like any centroid row and go
 * through the same matrix instructions as the scores they must equal; detection, location,
 * correction, strict mode, the detection threshold (ftk_fast_plan reports it) and the injection
 * hook are those of the register-resident fp32 kernels.
 * workspace: ftk_workspace_bytes(dtype, N, D, K, ft) bytes. */
ftk_status ftk_kmeans_assign_fast(ftk_dtype dtype, const void *X, const void *C, int64_t N, int32_t D,
                                  int32_t K, int32_t *labels, void *mindist /* nullable */,
                                  ftk_ft_mode ft, const ftk_fault *faults /* nullable */, int32_t n_faults,
                                  ftk_ft_stats *stats /* nullable */, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

/* (host) What ftk_assign_geometry and ftk_ft_thresholds report, for the reduced-precision path:
 * the extents fault descriptors are taken modulo, the detection threshold and the settlement band
 * (both as multiples of B_i, see ftk_ft_thresholds).  For 32 < D <= 128 band_coef and detect_coef are
 * upper bounds: the kernel's threshold is the rounding term plus ||x_i|| times the measured
 * truncation of the two-piece checksum rows, which is at most (and typically a tenth of) the 2^-16 *
 * 15 * max||c|| counted here.  Any output may be NULL. */
ftk_status ftk_fast_plan(ftk_dtype dtype, int64_t N, int32_t D, int32_t K, ftk_ft_mode ft,
                         ftk_geometry *geometry, double *detect_coef, double *band_coef);

/* Largest finite |x| over `count` elements, written as one double to out_absmax (device); NaN and
 * Inf elements are skipped.  ftk_kmeans_update needs it to fix the scale of its
 * order-independent accumulation. */
ftk_status ftk_absmax(ftk_dtype dtype, const void *X, int64_t count, double *out_absmax,
                      void *hip_stream);

/* Update step, Eq. (2), Sections 3.1.1-3.1.2 (sum the points of each cluster, then average).
 *   X [N x D], labels [N] in  : labels must lie in [0, K).
 *   C [K x D]             i/o : previous centroids in, new centroids out; rows of empty
 *                               clusters are left untouched.
 *   counts [K] int32      out : points per cluster.
 *   x_absmax              in  : device scalar from ftk_absmax over X, or NULL to have it
 *                               computed here (one more pass over X).
 * The result is bitwise reproducible from run to run: sums are accumulated in 64-bit fixed
 * point, which does not depend on the order of additions.
 * Accuracy: every coordinate is quantised once to a multiple of q = x_absmax * 2^-(61 - ceil(log2 N))
 * (fp32; at least 2^-50 x_absmax) or x_absmax * 2^-50 (fp64) before it is added, so a centroid
 * coordinate is off by at most q / 2 plus the final rounding to dtype, whatever its own
 * magnitude: one scale serves all features, and a feature whose values are many orders of
 * magnitude below the largest |x| of X keeps correspondingly fewer significant bits (for fp32
 * data and N = 2^20 the full 24 bits down to 2^-17 of the largest; for fp64 a feature 10^6
 * times smaller than the largest keeps about 31 bits).
 * X must be finite.  A NaN or Inf coordinate makes the centroid of the cluster its point is
 * labelled with unspecified (and, in the assignment, gives that point label 0 or any label in
 * range); all other clusters and points are unaffected, and nothing faults. */
ftk_status ftk_kmeans_update(ftk_dtype dtype, const void *X, const int32_t *labels, int64_t N,
                             int32_t D, int32_t K, void *C, int32_t *counts,
                             const double *x_absmax, void *workspace, size_t workspace_bytes,
                             void *hip_stream);

/* One Lloyd iteration (assignment, then update) carried out batch by batch: the single-pass idea of
 * Section 2.2 in the form this hardware allows.  The rows of X are taken in batches of `batch_rows`
 * points; each batch is assigned and, while it is still in the memory-side cache, added to the
 * running fixed-point sums; the centroids are averaged once after the last batch.  X is then read
 * from HBM once per iteration instead of twice, at the price of several launches per batch and of
 * a thinner grid per launch.  Results: labels and mindist as from ftk_kmeans_assign against the
 * incoming C; C and counts as from ftk_kmeans_update within its stated accuracy (the update always
 * runs on the per-workgroup table path here, so the last bits may differ from ftk_kmeans_update's).
 *   C [K x D]            i/o : centroids in, updated centroids out.
 *   x_absmax             in  : device scalar from ftk_absmax over X (required).
 *   batch_rows               : points per batch, at least N / 4096.
 * No fault tolerance on this path.  workspace: ftk_workspace_bytes(dtype, N, D, K, FTK_FT_OFF). */
ftk_status ftk_kmeans_step_batched(ftk_dtype dtype, const void *X, int64_t N, int32_t D, int32_t K, void *C,
                                   int32_t *labels, void *mindist /* nullable */, int32_t *counts,
                                   const double *x_absmax, int64_t batch_rows, void *workspace,
                                   size_t workspace_bytes, void *hip_stream);

/* The same update step protected by dual modular redundancy (Sections 2.3 and 4: the
 * memory-bound update is covered by duplicating its arithmetic and comparing).  With
 * ft != FTK_FT_OFF every arithmetic result of the step - conversion to fixed point, running
 * sums, member counts, table sums, scaling and division - is produced twice from the same
 * loaded operands and the two results are compared as integers before they leave the
 * registers (label-sorted path) or through a shadow total per workgroup (LDS-table path).
 *   DETECT           : a mismatch is counted (`detected`); the first result is used.
 *   CORRECT / STRICT : the affected run / workgroup pass is recomputed (`recomputed`; a pass
 *                      that mismatches again counts as `uncorrectable`), so the result equals
 *                      the fault-free one bit for bit.
 *   faults [n_faults] in : soft errors to inject into the first instruction stream of the
 *                      accumulating kernel: flip `bit` (mod 64) of the running sum / converted
 *                      operand number `reg` of lane `lane`, wave `wave`, workgroup `workgroup`,
 *                      after step `tile` of its row loop; extents from ftk_update_geometry.
 *                      With ft == FTK_FT_OFF they are injected unprotected.
 *   stats             i/o : injected / detected / recomputed / uncorrectable are added to. */
ftk_status ftk_kmeans_update_ft(ftk_dtype dtype, const void *X, const int32_t *labels, int64_t N,
                                int32_t D, int32_t K, void *C, int32_t *counts,
                                const double *x_absmax, ftk_ft_mode ft, const ftk_fault *faults,
                                int32_t n_faults, ftk_ft_stats *stats, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* Extents of the fault coordinates of ftk_kmeans_update_ft (rows_aligned16: whether X rows are
 * 16-byte aligned, i.e. X % 16 == 0 and D * element size % 16 == 0).  A register beyond what the last
 * 16 bytes of a row hold names one that they do. */
ftk_status ftk_update_geometry(ftk_dtype dtype, int64_t N, int32_t D, int32_t K,
                               int32_t rows_aligned16, ftk_geometry *out /* (host) */);

/* Lloyd loop, Section 2: `iters` times { assign ; update }, fixed iteration count.
 *   C_init [K x D]        in  : initial centroids, or NULL to take K distinct points of X
 *                               chosen by Floyd sampling driven by SplitMix64(seed)
 *                               (requires K <= N).
 *   C_out [K x D]         out : centroids after the last update.
 *   labels_out [N]        out : labels of the last assignment (taken against the centroids
 *                               before the last update).
 *   counts_out [K]        out : cluster sizes of that assignment.
 *   inertia_per_iter      out : (host, may be NULL) sum of mindist of every iteration;
 *                               when given, the call waits for the stream before returning.
 *   ft                        : mode of the assignment (checksums) and of the update (DMR).
 *   stats                 i/o : fault-tolerance counters summed over iterations, may be NULL. */
ftk_status ftk_kmeans_fit(ftk_dtype dtype, const void *X, int64_t N, int32_t D, int32_t K,
                          int32_t iters, uint64_t seed, const void *C_init, void *C_out,
                          int32_t *labels_out, int32_t *counts_out, double *inertia_per_iter,
                          ftk_ft_mode ft, ftk_ft_stats *stats, void *workspace,
                          size_t workspace_bytes, void *hip_stream);

/* The same loop with the assignment on the split-bf16 matrix path (ftk_kmeans_assign_fast):
 * fp32 data with D <= 128, D a multiple of 4, X 16-byte aligned.  Arguments as for
 * ftk_kmeans_fit, fault-tolerance mode (checksummed assignment, DMR update) and counters
 * included; workspace of ftk_workspace_bytes(dtype, N, D, K, ft) bytes. */
ftk_status ftk_kmeans_fit_fast(ftk_dtype dtype, const void *X, int64_t N, int32_t D, int32_t K,
                               int32_t iters, uint64_t seed, const void *C_init /* nullable */,
                               void *C_out, int32_t *labels_out, int32_t *counts_out,
                               double *inertia_per_iter /* (host) nullable */, ftk_ft_mode ft,
                               ftk_ft_stats *stats /* nullable */, void *workspace, size_t workspace_bytes,
                               void *hip_stream);

/* (host) K distinct indices in [0, N) by the seeded procedure ftk_kmeans_fit uses. */
ftk_status ftk_seeded_indices(uint64_t seed, int64_t N, int32_t K, int64_t *idx_host);

/* ---- rows sorted by label and back ---------------------------------------------------------
 * An assignment labels every row with its nearest centroid; a gate labels every token with the k experts it
 * likes best.  These calls bring the rows of one label together, so that what belongs to the label (an
 * inverted list, an expert's matrix) can be applied to them, bring the results back with weights, and
 * give the gradients of both.
 *   N tokens of D elements with k slots each, E experts; slot s = t * k + j belongs to token t.
 *   labels [N x k] int32: a slot whose label lies outside [0, E) is dropped: it takes no row and adds
 *   nothing anywhere, whatever its weight.  N = 0 is a valid, empty call.
 * Sorted rows: expert e has the rows [offsets[e], offsets[e + 1]), its slots in ascending order first, then
 * fill up to a multiple of `align`; rows beyond offsets[E] hold nothing either.  `rows` is the number of
 * sorted rows that the caller's arrays have, at least ftk_route_rows(N, k, E, align).
 *   order [rows] int32  : slot of a sorted row, -1 where it holds none
 *   pos [N x k] int32   : sorted row of a slot, -1 where it was dropped
 * Index arrays are device data that a call cannot check first: entries outside their range count as -1.
 * dtype: any.  Row arrays have unit stride along a row and a row stride (ldx, ... in elements, >= D).
 * Weights are float, for FTK_F64 double.  Sums are held in 32 bits (FTK_F64: 64), in ascending j, and rounded
 * once.  Everything is bitwise reproducible.
 * Limits: N * k + E * (align - 1) < 2^31, 1 <= E <= 8192, 1 <= k <= 64, 1 <= align <= 65536.
 * Up to FTK_ROUTE_FEW slots (N * k) no workspace is needed: NULL will do. */
#define FTK_ROUTE_FEW 1024
int64_t ftk_route_rows(int64_t N, int32_t k, int32_t E, int32_t align); /* -1: bad arguments */
size_t ftk_route_workspace_bytes(int64_t N, int32_t k, int32_t E);      /* 0: bad arguments */

/* Where every slot goes: offsets [E + 1], counts [E] (slots of every expert without the fill; may be NULL),
 * order [rows], pos [N x k], all int32 and out. */
ftk_status ftk_route_plan(const int32_t *labels, int64_t N, int32_t k, int32_t E, int32_t align,
                          int64_t rows, int32_t *offsets, int32_t *counts /* nullable */, int32_t *order,
                          int32_t *pos, void *workspace, size_t workspace_bytes, void *hip_stream);

/* out[p] = X[order[p] / k], times weights[order[p]] where weights are given; zero where order[p] is -1.
 *   X [N x D], out [rows x D].  out must not overlap X. */
ftk_status ftk_route_gather(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int32_t k, int32_t D,
                            const int32_t *order, const int32_t *pos, int64_t rows,
                            const void *weights /* nullable */, void *out, int64_t ldo, void *hip_stream);

/* ftk_route_plan and ftk_route_gather (without weights) in one call, for few slots in one launch. */
ftk_status ftk_route_dispatch(ftk_dtype dtype, const void *X, int64_t ldx, int32_t D, const int32_t *labels,
                              int64_t N, int32_t k, int32_t E, int32_t align, int64_t rows, int32_t *offsets,
                              int32_t *counts /* nullable */, int32_t *order, int32_t *pos, void *out,
                              int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream);

/* out[t] = sum over the slots of t of weights[t, j] * Y[pos[t, j]] (weights NULL: 1; then this is the gradient
 * of ftk_route_gather without weights).  A token all of whose slots were dropped gets zeros.
 *   Y [rows x D], out [N x D].  out must not overlap Y. */
ftk_status ftk_route_combine(ftk_dtype dtype, const void *Y, int64_t ldy, int64_t rows, const int32_t *pos,
                             const void *weights /* nullable */, int64_t N, int32_t k, int32_t D, void *out,
                             int64_t ldo, void *hip_stream);

/* Gradients of ftk_route_combine with weights: dY[pos[t, j]] = weights[t, j] * dOut[t] (zero in rows without a slot),
 * dweights[t, j] = <dOut[t], Y[pos[t, j]]> (zero for dropped slots; type of the weights).
 *   dOut [N x D], Y and dY [rows x D] (dY must not overlap Y or dOut). */
ftk_status ftk_route_combine_grad(ftk_dtype dtype, const void *dOut, int64_t ldg, const void *Y, int64_t ldy,
                                  const int32_t *order, const int32_t *pos, int64_t rows, const void *weights,
                                  int64_t N, int32_t k, int32_t D, void *dY, int64_t ldd, void *dweights,
                                  void *hip_stream);

/* ---- rows in microscaled 4-bit floating point, and products of them ---------------------------
 * The MXFP4 format of the OCP Microscaling Formats specification 1.0: 32 consecutive elements of a row share a power of two
 * 2^b, b = max(floor(log2 max|x|) - 2, -127), held as the byte b + 127; an element is sign, two bits of
 * exponent and one of mantissa, one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives: x / 2^b rounded
 * to the nearest, ties to the even code, beyond 6 to 6.  A block that holds an infinity or NaN gets the byte
 * 255 and stands for 32 NaN.
 * Packed rows are padded with zeros to Dp = D rounded up to 128 elements:
 *   codes [N x Dp / 2] bytes, 16-byte aligned: element 2i in the low half of byte i, 2i + 1 in the high half
 *   scales [N x Dp / 32] bytes, 4-byte aligned
 * dtype of dense rows: FTK_F32, FTK_BF16 or FTK_F16. */

/* Packs the N rows of X [N x D]; transpose != 0: the D columns, i.e. the rows of X^T (codes [D x Np / 2], scales
 * [D x Np / 32], Np = N rounded up to 128). */
ftk_status ftk_mx4_quantize(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int32_t D, int32_t transpose,
                            void *codes, void *scales, void *hip_stream);

/* out [N x D] of `dtype` from N packed rows of D elements, each value rounded once (FTK_F32, FTK_BF16: exact but for the
 * type's range). */
ftk_status ftk_mx4_dequantize(ftk_dtype dtype, const void *codes, const void *scales, int64_t N, int32_t D,
                              void *out, int64_t ldo, void *hip_stream);

/* The experts' products on packed rows: out[m, f] = sum_d A[src(m), d] * B[g(m) * F + f, d].
 *   A : N packed rows of D elements; B : E * F packed rows of D elements, E matrices of F rows.
 *   offsets [E + 1]  : expert e has the output rows [offsets[e], offsets[e + 1]) (device data, ascending, within
 *                      [0, M]); rows in front of the first one's and behind the last one's become zero.  NULL: E
 *                      must be 1 and has all rows.
 *   order [M], k     : src(m) = order[m] / k, and an output row whose order[m] is -1 becomes zero; NULL: src(m) = m.
 *   out [M x F]      : FTK_F32, FTK_BF16 or FTK_F16, row stride ldo.  N must be at least M where order is NULL.
 * Products of 4-bit elements are exact, sums are held in 32 bits and rounded once to out's type.
 * Limits: M < 2^31, F and D < 2^24, E <= 8192, E * F < 2^31. */
ftk_status ftk_mx4_matmul(ftk_dtype out_dtype, const void *a_codes, const void *a_scales, int64_t N,
                          const void *b_codes, const void *b_scales, int64_t M, int32_t F, int32_t D, int32_t E,
                          const int32_t *offsets /* nullable */, const int32_t *order /* nullable */, int32_t k,
                          void *out, int64_t ldo, void *hip_stream);

/* The same from dense rows X [N x D] of `dtype`, packed on the way exactly as ftk_mx4_quantize does; out has
 * their type.  workspace: ftk_mx4_workspace_bytes(N, D, M, E) bytes; where that is 0, as for few rows, NULL will do. */
ftk_status ftk_mx4_linear(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *b_codes,
                          const void *b_scales, int64_t M, int32_t F, int32_t D, int32_t E,
                          const int32_t *offsets /* nullable */, const int32_t *order /* nullable */, int32_t k,
                          void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream);
int64_t ftk_mx4_workspace_bytes(int64_t N, int32_t D, int64_t M, int32_t E); /* -1: bad arguments */

/* Sums over the rows of every expert, the gradient of the experts' matrices:
 *   out[e][f, d] = sum over p in [offsets[e], offsets[e + 1]) of A[f, p] * B[d, p]
 *   A : F packed rows of `rows` elements, B : D packed rows of `rows` elements (ftk_mx4_quantize with transpose of sorted
 *       rows, those without a slot zero); offsets on multiples of 128 (ftk_route_plan with align = 128 or a multiple; others
 *       are rounded down); NULL: E must be 1 and has all rows.
 *   out [E x F x D] contiguous, FTK_F32, FTK_BF16 or FTK_F16; experts without rows get zeros. */
ftk_status ftk_mx4_outer(ftk_dtype out_dtype, const void *a_codes, const void *a_scales, const void *b_codes,
                         const void *b_scales, int64_t rows, int32_t F, int32_t D, int32_t E,
                         const int32_t *offsets /* nullable */, void *out, void *hip_stream);

/* ---- a gate that learns ------------------------------------------------------------------------
 * Which k of E experts each of N rows goes to, from logits [N x E] (FTK_F32, FTK_BF16 or FTK_F16, row stride ldz):
 *   p = softmax of a row; labels [N x k]: its k largest logits in descending order, equal ones in ascending index;
 *   weights [N x k]: p of them, or with normalise != 0 the softmax over them alone; lse [N]: log of the sum of exponentials.
 * and how evenly the rows use the experts:
 *   counts [E + 1] : slots of every expert, and behind them T, the rows that took part
 *   probs [E]      : mean of p over those rows
 *   loss [1]       : E * sum_e counts[e] / (k T) * probs[e], 1 where all are used alike; 0 where T is.
 * An expert whose logit is -infinity is closed to the row: it is never chosen, and slots that find no expert get the label -1
 * (a dropped slot of ftk_route_plan) and the weight 0.  A row closed to all takes no part: lse -infinity.  A row with
 * a NaN or +infinity gets labels -1 and NaN weights, and makes probs and loss NaN.
 * Sums are held in 32 bits or more, in an order that N, E, k and dtype set: results are bitwise reproducible.
 * workspace: ftk_route_gate_workspace_bytes(N, E); up to FTK_ROUTE_GATE_FEW logits (N * E) none is needed: NULL will do.
 * Limits: 1 <= E <= 8192, 1 <= k <= 64, k <= E, N * k < 2^31.  N = 0 is a valid call (T = 0). */
#define FTK_ROUTE_GATE_FEW 16384
size_t ftk_route_gate_workspace_bytes(int64_t N, int32_t E); /* 0: bad arguments */
ftk_status ftk_route_gate(ftk_dtype dtype, const void *logits, int64_t ldz, int64_t N, int32_t E, int32_t k, int32_t normalise,
                          int32_t *labels, float *weights, float *lse, int32_t *counts, float *probs, float *loss,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/* dlogits [N x E] (type of the logits; may be the logits themselves) = gradient of sum(dweights * weights) + dloss * loss, labels and
 * counts held fixed.  dweights [N x k] or dloss [1] (device) may be NULL.  labels, weights, lse and counts as ftk_route_gate left
 * them (counts may have been summed over several calls, or processes, with equal E and k: the loss is then that of all their
 * rows). */
ftk_status ftk_route_gate_grad(ftk_dtype dtype, const void *logits, int64_t ldz, int64_t N, int32_t E, int32_t k,
                               int32_t normalise, const int32_t *labels, const float *weights, const float *lse,
                               const int32_t *counts, const float *dweights /* nullable */, const float *dloss /* nullable */,
                               void *dlogits, int64_t ldd, void *hip_stream);

/* ---- softmax cross entropy over many classes ------------------------------------------------------
 * Rows against the classes' vectors, the soft counterpart of the assignment: with bias_v = -||w_v||^2 / 2 a logit is the
 * assignment's score (Section 3.1.2) of a centroid.  The logits [N x V] are not kept.
 *   z_nv = scale * <x_n, w_v> + bias_v;   lse_n = log sum_v exp z_nv;   loss_n = lse_n - z_n,label_n
 *   X [N x D], W [V x D] of `dtype` (FTK_F32, FTK_BF16 or FTK_F16), row strides ldx and ldw; bias [V] or NULL: 0
 *   labels [N]: a row whose label lies outside [0, V) is ignored: nothing of it is looked at, loss and lse are 0
 *   loss, lse [N]
 * Logits, sums and lse are held in 32 bits (loss is off by half a step of lse); FTK_F32 operands (below 2^127) are taken to 24 bits.  W has to be finite.  A bias of
 * -infinity closes a class.  A row all of whose logits are -infinity has lse -infinity, a NaN loss and no gradient; a NaN or
 * +infinity among its logits makes a row's loss, lse and gradients NaN.  Results are bitwise reproducible.
 * workspace: ftk_xent_workspace_bytes(dtype, N, V, D, grad); it grows with N * max(D, 256), not with N * V: the classes go in pieces
 * of up to 256 MB (gradients, or W laid out anew: FTK_F32, or rows whose address, stride or length is no multiple of 16 bytes).
 * Limits: N, V < 2^31, D <= 2^20. */
int64_t ftk_xent_workspace_bytes(ftk_dtype dtype, int64_t N, int64_t V, int32_t D, int32_t grad); /* -1: bad arguments */
ftk_status ftk_xent(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *W, int64_t ldw, int64_t V, int32_t D,
                    const float *bias /* nullable */, double scale, const int32_t *labels, float *loss, float *lse,
                    void *workspace, size_t workspace_bytes, void *hip_stream);

/* Gradients of sum(dloss * loss), d_nv = dloss_n (exp(z_nv - lse_n) - [v = label_n]), zero for ignored rows:
 *   dX = scale * d W [N x D], dW = scale * d^T X [V x D] (type of the rows), dbias_v = sum_n d_nv [V]; each may be NULL,
 *   not all of them unless N = 0.
 * lse as ftk_xent left it; exp(z - lse) is off by half a step of lse, 2^-8 at most.  From |lse| = 2^17 on, where that would be more (masks of
 * the type's lowest value on all classes), the row's probabilities are divided by their own sum, which takes another pass over W for
 * every 64 rows that have such a one among them.
 * d is rounded to the rows' type (FTK_F32: not at all) before the products, and the gradients after them, which leaves those of 16-bit rows
 * off by 1.4 times a single rounding on average.  Every gradient is written once, in whole, and must not overlap an input. */
ftk_status ftk_xent_grad(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *W, int64_t ldw, int64_t V, int32_t D,
                         const float *bias /* nullable */, double scale, const int32_t *labels, const float *lse,
                         const float *dloss, void *dX /* nullable */, int64_t lddx, void *dW /* nullable */, int64_t lddw,
                         float *dbias /* nullable */, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- many weights updated at once ----------------------------------------------------------------
 * One AdamW step over a list of tensors, in place, one pass over each:
 *   g = grad_scale * grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2      (32 bits, every operation rounded)
 *   w = w - lr lr_scale (weight_decay w + m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps))
 * param: FTK_F32, FTK_BF16 or FTK_F16 (`dtype`); grad: FTK_F32 or the weights' type, for weights in 32 bits any of the three.
 * master: 32-bit weights beside 16-bit ones, which become the masters rounded; all tensors of a call have them or none has.
 *   Without them updates smaller than half a step of a 16-bit weight are lost.
 * state_bits 32: m and v are floats.
 * state_bits 8: m, v [count] codes and m_scales, v_scales [ceil(count / 32)].  32 consecutive elements share a power of
 *   two 2^b, held as the byte b + 127.  A code is exponent e (4 bits) over mantissa f (M bits: 3 for m, under a sign; 4 for v) and
 *   stands for f * 2^b where e = 0, else (2^M + f) * 2^(e - 1) * 2^b.  b is the least (>= -127) for which none of the block
 *   can be rounded out of range.  Numbers are rounded to one of their neighbours at random, the nearer one more often, so
 *   that the expected value is the number (rounded to the nearest, a state that changes by less than half a step would
 *   stay for ever); a positive v is never rounded to 0.  The random bits are a function of (seed, step, place in the
 *   list, element): a step is bitwise reproducible.  A block with an infinity or NaN gets the byte 255 and stands for 32 NaN.
 *   All zeros is the start of both kinds of state.
 * Tensors: any alignment of their element type, contiguous, apart from each other.  A tensor without grad (NULL), or of no
 * elements, is left as it is.  count <= 2^37.  Nothing is kept of the list: it may change from call to call. */
typedef struct {
    void *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scales, *v_scales; /* state_bits 8 */
    float *master;                /* nullable */
    int64_t count;
} ftk_adamw_tensor;
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    const float *lr_scale, *grad_scale; /* device scalars, may be NULL: 1 */
    const int64_t *step;                /* device scalar: number of this step, 1 for the first (counted by the caller) */
    uint64_t seed;
} ftk_adamw_options;
ftk_status ftk_adamw_step(ftk_dtype dtype, ftk_dtype grad_dtype, int32_t state_bits, const ftk_adamw_tensor *tensors /* (host) */,
                          int32_t n, const ftk_adamw_options *options /* (host) */, void *hip_stream);

/* What 8-bit states stand for: m_out[i], v_out[i] [count] of `dtype`, rounded once (exact in FTK_F32 and FTK_BF16 but for the
 * type's range).  Takes m, v, m_scales, v_scales and count of the list's tensors.  m_out, v_out: lists (host) of n pointers. */
ftk_status ftk_adamw_moments(ftk_dtype dtype, const ftk_adamw_tensor *tensors /* (host) */, int32_t n, void *const *m_out /* (host) */,
                             void *const *v_out /* (host) */, void *hip_stream);

/* Profiling aid for benchmarks.  While enabled, every ftk_kmeans_assign call brackets its main
 * contraction kernel (not the small norm / refine kernels around it; on the scan path: the scan with
 * its preparation and settlement; in a small unprotected fit: the one launch of an iteration) with a pair of HIP events
 * recorded on the call's stream.  ftk_profile_read waits for all recorded pairs, returns the
 * summed kernel time in milliseconds and the number of launches since the last read (host
 * pointers), and releases the events.  Not thread-safe; creates events, so keep it out of
 * throughput timing loops. */
ftk_status ftk_profile_enable(int32_t on);
ftk_status ftk_profile_read(double *total_ms, int64_t *launches);

/* Hook for the shape-sweep / tuning tool (the counterpart of the paper's kernel selection,
 * Section 3.2: measure the candidates per problem shape, keep the fastest).  Forces, for every
 * later call of this process, the choices the library otherwise makes by rule; -1 restores a
 * rule.  Every forced choice computes the same results.
 *   assign_variant : 0 = generic kernel, 1 = the register-resident kernels where they apply
 *                    (fp32, 16-byte aligned rows: the small-D kernel for D <= 32, the mid-D
 *                    kernel for 32 < D <= 128 with D a multiple of 4)
 *   generic_tiles  : centroid tiles per chunk of the generic kernel, 1, 2, 4 or 8 (8: one point
 *                    tile per wave instead of two; chosen by rule only for fp64 with long rows)
 *   update_path    : 0 = per-workgroup LDS tables, 1 = label-sorted gather
 * Process-wide and not synchronised: set it while no call is in flight.  The workspace size
 * does not depend on it. */
ftk_status ftk_tuning_override(int32_t assign_variant, int32_t generic_tiles, int32_t update_path);

const char *ftk_last_error(void);
const char *ftk_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FTKMEANS_H */
