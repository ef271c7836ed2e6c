/*
 * externd.h -- C ABI of the MI355X (gfx950) ExTernD factorizer.
 *
 * ExTernD approximates a matrix A (m x n) as A ~= B diag(D) C with ternary
 * factors B in {-1,0,1}^{m x k}, C in {-1,0,1}^{k x n} and real scales D,
 * k = mu * min(m, n) (paper: "ExTernD: Expanded-Rank Ternary
 * Decomposition", Sec. 2.1, Eq. (1)).  Components are extracted by greedy
 * alternating least squares with sequential deflation (Sec. 2.3), in blocks
 * of b components with decorrelated least-squares targets (Sec. 2.4,
 * Eq. (3)) and a joint exact scale solve (Eq. (4)); optionally with
 * per-column importance weights (Sec. 2.5; lambda = 0, or any lambda >= 0
 * through externd_factorize_ex).
 *
 * Conventions for every entry point:
 *  - "device" pointers are HIP device memory on the current device (for
 *    example torch.cuda tensor data pointers); "host" pointers are ordinary
 *    CPU memory.
 *  - Matrices are row-major and dense (leading dimension = column count).
 *  - The caller owns every buffer.  The library keeps no pointer to a
 *    caller buffer after a call returns and allocates no device memory;
 *    calls on distinct workspaces and streams are independent.  Calls
 *    sharing a workspace must be ordered (same stream or synchronised by the
 *    caller).  The one piece of global state is the fixed device scratch of
 *    externd_apply_noalloc (below), one copy per device.
 *  - `stream` is a hipStream_t (NULL = the default stream).  All device work
 *    is enqueued on it.
 *  - Errors are returned as negative status codes; no exception crosses the
 *    ABI.  Argument errors are detected on the host before any device work
 *    is enqueued.  On error the contents of output buffers are unspecified
 *    (host energy outputs are set to NaN where given).
 *
 * Packed trit format (B and C outputs): 2 bits per element, element j of a
 * row in byte (j >> 2) at bits 2*(j & 3) .. 2*(j & 3)+1; bit 0 = nonzero,
 * bit 1 = negative: 00 -> 0, 01 -> +1, 11 -> -1 (10 is never written).
 * Each row is padded to a whole byte with zero bits.
 */
#ifndef EXTERND_H
#define EXTERND_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EXTERND_OK            0
#define EXTERND_EINVAL       -1  /* bad scalar argument or NULL required pointer        */
#define EXTERND_ENONFINITE   -2  /* NaN/Inf in A (detected on the device)               */
#define EXTERND_EWORKSPACE   -3  /* workspace smaller than externd_workspace_bytes()    */
#define EXTERND_EHIP         -4  /* HIP runtime or launch failure                       */
#define EXTERND_EUNSUPPORTED -5  /* shape outside the supported range                   */
#define EXTERND_ESYNC        -6  /* a bounded wait between the workgroups of one kernel
                                    launch ran out (the U-step's row groups and the
                                    V-step's last row group of each column tile wait for
                                    the inverse Gram of the same launch, and in blocks
                                    wider than 64 the workgroups that build that inverse
                                    wait for each other; at most ten seconds, so that
                                    another stream's kernel may hold the GPU meanwhile);
                                    the factors of such a call are not to be used       */
#define EXTERND_ESCRATCH     -7  /* the call needs more than the fixed device scratch of
                                    an allocation-free entry point                       */

/* Largest effective block width the kernels handle (four quarters of 64
 * components; the paper's default b = 256, Sec. 2.4).  A call whose
 * effective width (externd_effective_block) exceeds it returns
 * EXTERND_EUNSUPPORTED before any device work; nothing is clamped.
 * Effective widths above 64 run the block as quarters coupled through
 * their Gram inverses and the joint solve; refinement sweeps and the
 * safeguard accept effective widths up to 64 only.                      */
#define EXTERND_MAX_BLOCK 256

/* Ridge of the decorrelated targets, Eq. (3): eps = EXTERND_RIDGE_REL *
 * trace(G) / bb for each Gram matrix G of a block of bb components.      */
#define EXTERND_RIDGE_REL 1e-6
/* Guard of the joint scale solve, Eq. (4): (M + delta I) d = g with
 * delta = EXTERND_SCALE_GUARD_REL * trace(M) / bb.                       */
#define EXTERND_SCALE_GUARD_REL 1e-12

/* Human-readable name of a status code (static string). */
const char* externd_strerror(int status);

/* Inner rank k = floor(mu * min(m, n) + 0.5) (Sec. 2.1); -1 if k < 1 or
 * the arguments are invalid.                                             */
int64_t externd_rank(int64_t m, int64_t n, double mu);

/* Block width actually used: min(block, floor(min(m, n) / 8)), at least
 * 1 (Sec. 2.4 caps b at min(m, n) / 8).  The factorizing entry points
 * return EXTERND_EUNSUPPORTED when it exceeds EXTERND_MAX_BLOCK.  -1 on
 * invalid arguments.                                                     */
int32_t externd_effective_block(int64_t m, int64_t n, int32_t block);

/* Device workspace, in bytes, for an m x n matrix and inner rank k:
 * k = externd_rank(m, n, mu) for externd_factorize, k = 0 for the step
 * entry points.  Independent of block and of whether weights are given:
 * sized for blocks of EXTERND_MAX_BLOCK components, 4 m n bytes for the
 * fp32 residual plus about 5.5 kB per row and (2 + 2 gv) kB per column
 * (gv <= 8 row groups of the V-step's partial contractions) and under
 * 16 MB of fixed buffers.  0 on invalid arguments or unsupported shapes. */
size_t externd_workspace_bytes(int64_t m, int64_t n, int64_t k);

/*
 * externd_factorize -- full greedy block-ALS factorization (Sec. 2.3-2.5).
 *
 *  A          device, fp32 m x n, read only.
 *  m, n       1 <= m <= 2^26, 1 <= n <= 2^20, and with both rounded up to
 *             multiples of 32 their product below 2^31 (else
 *             EXTERND_EUNSUPPORTED).
 *  mu         inner-rank multiplier, k = externd_rank(m, n, mu) >= 1.
 *  tau        threshold scale of T_tau, Eq. (2); finite, >= 0.
 *  block      requested block width b >= 1 (see externd_effective_block;
 *             block = 1 is the sequential algorithm of Sec. 2.3).  An
 *             effective width above EXTERND_MAX_BLOCK (256) is
 *             EXTERND_EUNSUPPORTED.
 *  iters      ALS iterations per block, >= 1; one iteration is a V-step
 *             followed by a U-step (Sec. 2.3 order).
 *  importance device fp32[n] per-column weights h (finite, >= 0, max > 0),
 *             or NULL for the plain Frobenius objective.  h~ = h / max(h).
 *  B_packed   device, m rows of ceil(k/4) bytes (packed trits, B[:, i]).
 *  C_packed   device, k rows of ceil(n/4) bytes (packed trits, C[i, :]).
 *  D          device fp32[k].
 *  energy     host, out: E = 1 - ||A - B diag(D) C||^2 / ||A||^2 (Sec. 2.1)
 *             as tracked on the device residual.
 *  energy_w   host, out (may be NULL): weighted energy
 *             1 - sum_j h~_j ||R_:j||^2 / sum_j h~_j ||A_:j||^2;
 *             equals energy when importance is NULL.
 *  energy_curve, energy_w_curve
 *             host, out (may be NULL): E (resp. weighted E) after each
 *             block, ceil(k / b_eff) doubles.
 *  workspace  device, >= externd_workspace_bytes(m, n, k) bytes, 256-byte
 *             aligned.
 *  stream     hipStream_t or NULL.
 *
 * Enqueues all work on `stream` and synchronises that stream before
 * returning (energies are host outputs).  Deterministic: identical inputs
 * give bit-identical outputs.
 */
int externd_factorize(const float* A, int64_t m, int64_t n, double mu, double tau,
                      int32_t block, int32_t iters, const float* importance,
                      uint8_t* B_packed, uint8_t* C_packed, float* D,
                      double* energy, double* energy_w,
                      double* energy_curve, double* energy_w_curve,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * externd_factorize_ex -- externd_factorize with the two options of the
 * method that the plain call fixes: the lambda of the importance weights
 * and the single-entry safeguard.
 *
 *  lambda     finite, >= 0: h~ = h / max(h) + lambda (Sec. 2.5; lambda
 *             interpolates between the importance-weighted objective at 0
 *             and the plain one as it grows).  Ignored when importance is
 *             NULL.  lambda = 0 gives externd_factorize's result bit for bit.
 *  safeguard  0 or 1.  1: the block form of Proposition 2's augmented step
 *             (Appendix A).  After each block's Eq. (4) solve, the objective
 *             the block removes, 2 d^T g - d^T M d, is compared with the
 *             largest squared residual entry R_ij^2 (the first in row-major
 *             order on ties); when the entry is strictly larger the block
 *             becomes u = e_i, v = sign(R_ij) e_j, d = |R_ij| followed by
 *             zero components, which removes R_ij exactly.  Every block then
 *             removes at least ||R||^2 / (m n).  Plain objective only:
 *             safeguard = 1 with importance != NULL is EXTERND_EINVAL.  When
 *             it never fires the outputs equal those of externd_factorize.
 *  safeguard_fired  host, out (may be NULL): blocks replaced.
 * Other arguments, workspace size, status codes and synchronisation as
 * externd_factorize.
 */
int externd_factorize_ex(const float* A, int64_t m, int64_t n, double mu, double tau, int32_t block, int32_t iters,
                         const float* importance, double lambda, int32_t safeguard, uint8_t* B_packed,
                         uint8_t* C_packed, float* D, double* energy, double* energy_w, double* energy_curve,
                         double* energy_w_curve, int64_t* safeguard_fired, void* workspace, size_t workspace_bytes,
                         void* stream);

/*
 * externd_factorize_to_energy -- the factorization stopped at an energy
 * target (the paper chooses mu per matrix so that a target accuracy is met
 * exactly, Sec. 1 and Sec. 3; greedy deflation makes every prefix of the
 * components the same as in a longer run, Sec. 2.1).
 *
 *  mu_max         k_max = externd_rank(m, n, mu_max) components at most.
 *  target_energy  finite; after each block the energy E (or, with
 *                 importance, the weighted energy E_w) is compared with
 *                 it, and extraction stops at the first block that
 *                 reaches it (or at k_max).
 *  k_used         host, out: components extracted, a multiple of the
 *                 effective block width, or k_max.
 *  B_packed, C_packed, D, workspace: sized for k_max as in
 *                 externd_factorize; components past k_used are zero.
 *  energy, energy_w: after k_used components.  energy_curve,
 *                 energy_w_curve (may be NULL): room for ceil(k_max / b)
 *                 entries, the first ceil(k_used / b) are written.
 * Other arguments, status codes and synchronisation as externd_factorize.
 * Each block adds one small device-to-host read of the energy history.
 */
int externd_factorize_to_energy(const float* A, int64_t m, int64_t n, double mu_max, double target_energy,
                                double tau, int32_t block, int32_t iters, const float* importance,
                                uint8_t* B_packed, uint8_t* C_packed, float* D, int64_t* k_used, double* energy,
                                double* energy_w, double* energy_curve, double* energy_w_curve, void* workspace,
                                size_t workspace_bytes, void* stream);

/*
 * externd_factorize_refined -- externd_factorize followed by refinement
 * sweeps (Sec. 2.4: after extraction each block is added back to the
 * residual, fitted again and deflated again, which raises energy
 * monotonically).
 *
 * A sweep revisits the blocks in extraction order.  A revisit forms
 * R' = R + U diag(d) V^T, runs `iters` V-step/U-step iterations of Eq. (3)
 * warm-started from the block's current U, and solves Eq. (4) for the new
 * scales d'.  The new block replaces the old one (in B_packed, C_packed
 * and D) only when the objective it removes from R', 2 d'^T g' - d'^T M' d'
 * (weighted when importance is given), exceeds what the old block removes,
 * ||R'||^2 - ||R||^2; otherwise the old block is deflated again and the
 * outputs keep it.  No revisit therefore increases the objective beyond the
 * rounding of the fp32 residual.
 *
 *  sweeps          >= 0 (0 gives the result of externd_factorize).
 *  energy, energy_w  host, out: after the last sweep.
 *  energy_curve, energy_w_curve  host, out (may be NULL): the extraction's
 *                  per-block curve, as in externd_factorize.
 *  sweep_energy, sweep_energy_w  host, out (may be NULL): E and weighted E
 *                  after each sweep (`sweeps` doubles each).
 *  accepted        host, out (may be NULL): revisits that replaced their
 *                  block, out of sweeps * ceil(k / b_eff).
 * Other arguments, workspace size, status codes and synchronisation as
 * externd_factorize.  Each sweep adds one small device-to-host read.
 */
int externd_factorize_refined(const float* A, int64_t m, int64_t n, double mu, double tau, int32_t block,
                              int32_t iters, int32_t sweeps, const float* importance, uint8_t* B_packed,
                              uint8_t* C_packed, float* D, double* energy, double* energy_w, double* energy_curve,
                              double* energy_w_curve, double* sweep_energy, double* sweep_energy_w,
                              int64_t* accepted, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Inference with a factorization (Sec. 2.6 cost model): for each of nb
 * input vectors x (rows of X), y = B (diag(D) (C x)), computed on the packed
 * trits in a fixed order (deterministic).
 *  - One vector with n, k <= 65536: integer matrix cores.  x and the
 *    intermediate t = diag(D) C x enter as 48-bit fixed-point vectors (one
 *    power-of-two scale each: x's from max |x|, t's from the bound
 *    max |D| sum_j |x_j|), so every product and sum is exact; the error is
 *    that of the two conversions and the final rounding: at most
 *    u |y| + 2^-46 [ (|B| (|D| (|C| 1))) max|x| + (|B| 1) max|D| sum|x| ]
 *    per output, u = 2^-24 (entries of x within 2^22 of max |x| convert
 *    exactly).  With n or k above 10240 no entry is rounded in conversion: a
 *    vector is summed exactly (in groups of 38 binades, added in fp64) or,
 *    where its side is small, in fp64, and only t and y are rounded, to fp32:
 *    u (|y| + |B| |t|) + (n + k + 4) 2^-53 |B| (|D| (|C| |x|)), whatever the
 *    largest entry.  A NaN or infinite entry of x or D makes every output NaN.
 *  - Otherwise one vector runs on fp32 FMA and two or more on bf16 matrix
 *    cores with exact operands (trits are exact in bf16; every fp32 vector
 *    entry is split exactly into three bf16 parts), with fp32 sums: at most
 *    (n + k + 4) u (|B| (|D| (|C| |x|))) per output, for finite inputs whose
 *    nonzero entries are fp32 normals.
 *
 *  B_packed   device, m rows of ceil(k/4) bytes; C_packed device, k rows of
 *             ceil(n/4) bytes; D device fp32[k] -- as written by
 *             externd_factorize (or _to_energy, whose zero components
 *             contribute nothing).  On the matrix-core path, rows of
 *             any length at any byte address take whole-word loads.
 *  X          device fp32, nb x n row-major.  Y device fp32, nb x m
 *             row-major (out).
 *  nb         1 <= nb <= EXTERND_APPLY_MAX_BATCH.
 *  workspace  device, >= externd_apply_workspace_bytes(m, n, k, nb) bytes,
 *             256-byte aligned.  nb = 1: the intermediate diag(D) C x
 *             (n, k <= 10240: its six 8-bit digit planes, 1536 bytes per
 *             256 entries, and an exponent word; else 4 k bytes).  nb >= 2: its bf16 parts (6 nb k bytes) and
 *             partial sums over slices of the contracted dimensions (at
 *             most nb max(n, m) k / 32 bytes, rounded up to whole row
 *             groups).
 * Asynchronous on `stream`.  m, n, k <= 2^31 (else EXTERND_EUNSUPPORTED).
 */
#define EXTERND_APPLY_MAX_BATCH 8
size_t externd_apply_workspace_bytes(int64_t m, int64_t n, int64_t k, int32_t nb);  /* 0 on invalid arguments */
int externd_apply(const uint8_t* B_packed, const uint8_t* C_packed, const float* D, int64_t m, int64_t n,
                  int64_t k, const float* X, int32_t nb, float* Y, void* workspace, size_t workspace_bytes,
                  void* stream);

/*
 * externd_apply without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, arithmetic, results
 * (bit for bit) and status codes as externd_apply, with the workspace held
 * in a fixed device array of the library instead:
 *  - at most EXTERND_APPLY_NOALLOC_MAX_BYTES, i.e.
 *    externd_apply_workspace_bytes(m, n, k, nb) <= that bound (m = 9728,
 *    n = 2560, k = 7680 takes 5.0 MB at nb = 8, 31 kB at nb = 1); larger
 *    calls return EXTERND_ESCRATCH before any device work;
 *  - the array is per device: the current device's copy is used, and the
 *    stream must belong to the current device.  Each device keeps its copy
 *    until the process ends.  The first call on a device looks up the
 *    array's address (hipGetSymbolAddress); no call allocates or frees
 *    device memory;
 *  - every call on a device shares that device's array: calls that overlap
 *    on one device (concurrent streams, or several host threads without
 *    ordering) race and give unspecified results.  Calls ordered on one
 *    stream are safe; nothing needs to be cleared between calls (every
 *    entry a call reads is written earlier in the same call).
 */
#define EXTERND_APPLY_NOALLOC_MAX_BYTES (8u << 20)
int externd_apply_noalloc(const uint8_t* B_packed, const uint8_t* C_packed, const float* D, int64_t m, int64_t n,
                          int64_t k, const float* X, int32_t nb, float* Y, void* stream);

/* Kernel classes timed by externd_factorize_timed. */
#define EXTERND_KCLASS_VSTEP   0  /* V-step contraction P = U^T R (+ Gram of U, inverse) */
#define EXTERND_KCLASS_USTEP   1  /* U-step contraction Q = R diag(h~) V (+ Gram of V)  */
#define EXTERND_KCLASS_DEFLATE 2  /* deflation R -= U diag(d) V^T (+ column energies)   */
#define EXTERND_KCLASS_VTARGET 3  /* V-step target Y = G_U^{-1} P and its statistics    */
#define EXTERND_KCLASS_UTARGET 4  /* U-step target Z = Q G_V^{-1} and its statistics    */
#define EXTERND_KCLASS_SEQ     5  /* the one-launch sequential path (block width 1 on a
                                     small matrix: every launch is timed)              */
#define EXTERND_KCLASS_TERNV   6  /* V = T_tau(Y^T) per component, Eq. (2)            */
#define EXTERND_KCLASS_TERNU   7  /* U = T_tau(Z) per component, Eq. (2) (+ g = diag(U^T Q)
                                     in the last U-step of a block)                     */
#define EXTERND_KCLASS_COUNT   8

typedef struct {
  double total_ms[EXTERND_KCLASS_COUNT];  /* summed durations of the timed launches */
  int64_t launches[EXTERND_KCLASS_COUNT]; /* number of timed launches of each class */
  int64_t issued[EXTERND_KCLASS_COUNT];   /* number of launches of each class       */
} externd_kernel_times;

/* Launches of each class timed by externd_factorize_timed: one in every
 * EXTERND_TIMING_STRIDE, evenly spread over the call.                    */
#define EXTERND_TIMING_STRIDE 16

/* externd_factorize with HIP events recorded on `stream` around a sample
 * of the launches of the kernel classes above (every
 * EXTERND_TIMING_STRIDE-th launch of a class; the events are created
 * without system-scope fences, so a timed launch ends without an L2
 * write-back, and add a small host-side cost per timed launch).  `times`
 * (host, required) receives the summed durations, the number of timed
 * launches and the number of all launches of each class.  Same outputs and
 * status codes as externd_factorize.                                     */
int externd_factorize_timed(const float* A, int64_t m, int64_t n, double mu, double tau,
                            int32_t block, int32_t iters, const float* importance,
                            uint8_t* B_packed, uint8_t* C_packed, float* D,
                            double* energy, double* energy_w,
                            double* energy_curve, double* energy_w_curve,
                            void* workspace, size_t workspace_bytes, void* stream,
                            externd_kernel_times* times);

/*
 * Step entry points: one step each of the block ALS on caller-given state,
 * for per-step parity checks.  They share the kernels of
 * externd_factorize.  Block matrices are row-major with bb columns:
 * U is m x bb int8 in {-1,0,1}, V is n x bb int8.  1 <= bb <= EXTERND_MAX_BLOCK.
 * Every pointer except `h` / `*_or_null` outputs is required.  These calls
 * are asynchronous on `stream`.
 */

/* Initial U of a block (paper silent; reading: the residual columns with
 * the bb largest h~_j ||R_:j||^2, ties to the smaller index, are
 * ternarized with T_tau, Eq. (2)).  J_out: device int32[bb], the chosen
 * column indices in descending order of weighted energy.                 */
int externd_step_init(const float* R, int64_t m, int64_t n, const float* h, int32_t bb,
                      double tau, int8_t* U_out, int32_t* J_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/* V-step of Eq. (3): Y = (U^T U + eps I)^{-1} U^T R, V[:, c] = T_tau(Y[c, :]).
 * V_out device int8 n x bb; Y_out_or_null device fp64 bb x n.            */
int externd_step_vstep(const float* R, int64_t m, int64_t n, const int8_t* U, int32_t bb,
                       double tau, int8_t* V_out, double* Y_out_or_null,
                       void* workspace, size_t workspace_bytes, void* stream);

/* U-step of Eq. (3) with the weighting of Sec. 2.5:
 * Q = R diag(h~) V, Z = Q (V^T diag(h~) V + eps I)^{-1}, U[:, c] = T_tau(Z[:, c]).
 * h may be NULL (h~ = 1).  U_out device int8 m x bb; Q_out_or_null and
 * Z_out_or_null device fp64 m x bb.                                      */
int externd_step_ustep(const float* R, int64_t m, int64_t n, const int8_t* V, int32_t bb,
                       double tau, const float* h, int8_t* U_out,
                       double* Q_out_or_null, double* Z_out_or_null,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Joint scale solve, Eq. (4): [(U^T U) o (V^T diag(h~) V) + delta I] d =
 * diag(U^T Q) with Q = R diag(h~) V (device fp64 m x bb, as returned by
 * externd_step_ustep).  d_out device fp64[bb].                           */
int externd_step_scale(const int8_t* U, const int8_t* V, const double* Q, int64_t m,
                       int64_t n, int32_t bb, const float* h, double* d_out,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Block deflation R <- R - U diag(d) V^T (Sec. 2.4), in place on the
 * device fp32 m x n matrix R, with d rounded to fp32 (as stored in D).
 * colnorm2_out device fp64[n] (may be NULL): ||R_:j||^2 after the update;
 * fro2_out device fp64[1] (may be NULL): ||R||_F^2 after the update.    */
int externd_step_deflate(float* R, int64_t m, int64_t n, const int8_t* U, const int8_t* V,
                         const double* d, int32_t bb, double* colnorm2_out, double* fro2_out,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Operators of decoding: what runs between and behind the projections that
 * externd_apply evaluates.  Rotary positions turn q and k, a cache in 4 bits
 * holds k and v, attention reads it, and the log probabilities of given
 * tokens judge the result (perplexity).
 *
 * Conventions, besides those at the top: `dtype` is one of the codes below
 * and holds for every array of that type in the call; strides count elements;
 * the innermost dimension of every array is dense.  All calls are
 * asynchronous on `stream`, allocate nothing and may be captured into a
 * graph.  Device contents that the host cannot see (positions, lengths, page
 * numbers, targets) never lead a kernel outside its arrays: what they would
 * reach there is left out as each call says.  Outputs are bit-identical from
 * run to run.
 */
#define EXTERND_F32  0
#define EXTERND_BF16 1
#define EXTERND_F16  2

/* Rotary frequencies, on the host (no device work).  Pair i of rot_dim / 2
 * turns by theta_i = base^(-2 i / rot_dim) radians a position.
 *  scaling  EXTERND_ROPE_PLAIN: as above.
 *           EXTERND_ROPE_LINEAR: theta_i / factor (positions interpolated).
 *           EXTERND_ROPE_BASE: base * factor^(rot_dim / (rot_dim - 2)), so that
 *           the slowest pair is interpolated and the fastest is not.
 *           EXTERND_ROPE_PARTS: with r_i = original_length theta_i / 2 pi turns
 *           in the trained context and g_i = clamp((r_i - beta_slow) /
 *           (beta_fast - beta_slow), 0, 1): theta_i (g_i + (1 - g_i) / factor);
 *           amplitude 0.1 ln(factor) + 1.
 *  freqs    host, out: rot_dim / 2 words, theta_i in units of 2^-64 turns.
 *  amplitude  host, out (may be NULL): the factor on the turned entries.
 * rot_dim even, 2 .. 1024; base > 1; factor >= 1; original_length >= 1 and
 * beta_fast > beta_slow for PARTS (ignored otherwise).  Any other word may be
 * used as a frequency too: a position p turns pair i by p freqs[i] mod 2^64,
 * which is exact at every position.                                       */
#define EXTERND_ROPE_PLAIN  0
#define EXTERND_ROPE_LINEAR 1
#define EXTERND_ROPE_BASE   2
#define EXTERND_ROPE_PARTS  3
int externd_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                               int64_t original_length, double beta_fast, double beta_slow, uint64_t* freqs,
                               double* amplitude);

/* Rotary positions of q and (k may be NULL) k: with phi = positions[t] theta_i,
 *   a' = amplitude (a cos phi - b sin phi),  b' = amplitude (b cos phi + a sin phi)
 * for the pairs (a, b) = entries (i, i + rot_dim / 2) of each head
 * (interleaved = 0) or (2 i, 2 i + 1) (interleaved = 1), i < rot_dim / 2;
 * entries from rot_dim on are copied.  inverse = 1 turns by -phi: the gradient
 * of the same call.  The arithmetic is fp32, rounded once to dtype.
 *  q, q_out   device, tokens x heads_q x head_dim with the given strides; q_out
 *             may be q with the same strides (in place), and no other overlap.
 *  positions  device int64[tokens], any value; freqs device uint64[rot_dim / 2].
 * head_dim 2 .. 1024, rot_dim even, 2 .. head_dim; tokens 0 is a valid call;
 * tokens < 2^31, heads_q + heads_k <= 65535.                                */
int externd_rotary(const void* q, void* q_out, int64_t q_token_stride, int64_t q_head_stride,
                   int64_t q_out_token_stride, int64_t q_out_head_stride, int32_t heads_q, const void* k,
                   void* k_out, int64_t k_token_stride, int64_t k_head_stride, int64_t k_out_token_stride,
                   int64_t k_out_head_stride, int32_t heads_k, int32_t dtype, int64_t tokens, int32_t head_dim,
                   int32_t rot_dim, int32_t interleaved, int32_t inverse, const int64_t* positions,
                   const uint64_t* freqs, float amplitude, void* stream);

/*
 * The cache in 4 bits.  Pages of page_tokens tokens (a power of two, 16 ..
 * 1024); a page holds, for each of heads_kv heads, externd_kv4_page_bytes()
 * bytes: with P = page_tokens, D = head_dim (64, 128 or 256), H = D / 2,
 *   K codes  [P][H]          byte i: channel i (low nibble), i + H (high)
 *   V codes  [P / 16][H][16] the same bytes, tokens of a block side by side
 *   words    [P][2][D / 64]  uint16, K's then V's, one per 64 channels: an
 *                            fp16 scale s whose low four bits hold the zero
 *                            point z.  A value is s (code - z).
 * For 64 values x with lo = min(x, 0), hi = max(x, 0): s is (hi - lo) / 15
 * rounded up to seven significant bits (to a multiple of 2^-20 below 2^-14),
 * at most 4352; z = round(-lo / s), code = round(x / s) + z in 0 .. 15.  Every
 * value is exactly an fp16 number, and within s / 2 of x (s (1 + 2^-20) / 2
 * with the rounding of x / s) while hi - lo <= 65280.  64 values with an
 * infinity or a NaN among them are all held as NaN.
 *
 * Sequences: the cache belongs to `batch` sequences.  Device int32 lens[batch]
 * is the number of tokens in each, the new ones of this step included; token
 * position p of sequence b is in page table[b table_pages + p / P] at p % P.
 * Device int32 starts[batch + 1] (rising from 0 to `tokens`) says where the
 * new tokens of each sequence are in the call's arrays; NULL: one token each
 * (tokens = batch).  The new tokens are the last ones: token i of a sequence's
 * n new ones is at position lens - n + i, whatever the table holds.  Positions
 * below 0 and from table_pages P on have no place: not stored, read as 0 and
 * seen by no query, though a query may be there.  Page numbers outside
 * [0, num_pages) name pages without tokens.
 */
size_t externd_kv4_page_bytes(int32_t head_dim, int32_t page_tokens);  /* of one head; 0 on invalid arguments */

/* Stores the new tokens' k and v (device, tokens x heads_kv x head_dim).
 * Tokens whose position or page is none are not stored.  cache: device, 16-byte
 * aligned, num_pages x heads_kv x externd_kv4_page_bytes() bytes.  Two tokens
 * of one call must not share a place.  num_pages, tokens heads_kv < 2^31,
 * (tokens / 16 + 2 batch) heads_kv < 2^25.                                 */
int externd_kv4_append(void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim, int32_t page_tokens,
                       const void* k, const void* v, int32_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                       int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, int32_t batch,
                       const int32_t* starts, const int32_t* lens, const int32_t* table, int64_t table_pages,
                       void* stream);

/* The values held for the new tokens (with starts over whole sequences: for
 * all tokens), dense and 16-byte aligned, as dtype; 0 where a token has no
 * place.                                                                   */
int externd_kv4_read(const void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim, int32_t page_tokens,
                     void* k, void* v, int32_t dtype, int64_t tokens, int32_t batch, const int32_t* starts,
                     const int32_t* lens, const int32_t* table, int64_t table_pages, void* stream);

/* Attention of the new tokens over the cache: with the values k^, v^ held,
 * for query head h (cache head h heads_kv / heads_q) of a token at position p,
 *   x_j = scale q . k^_j,  out = sum_j softmax(x)_j v^_j,  lse = ln sum_j exp x_j
 * over the positions j <= p, and j > p - window where window > 0.  No such j
 * (an empty sequence, a position below 0, pages without tokens): out 0 and
 * lse -infinity.
 *  q          device, tokens x heads_q x head_dim; out device, dense, the same,
 *             at any entry of its type.
 *  lse        device fp32, tokens x heads_q, or NULL.
 *  max_new    the largest number of new tokens of one sequence, or more.
 *  max_len    the largest length, or more; 0: not known.  Both only choose
 *             the launch: results hold whatever they are.
 *  heads_q a multiple of heads_kv, heads_q / heads_kv <= 64; scale finite;
 *  window >= 0; batch <= 65535, tokens heads_q < 2^31 - 1024, and with R the
 *  lesser of table_pages page_tokens and 2^31 - 1, (R / 64 + 16) heads_kv < 2^31.
 *  workspace  device, >= externd_kv4_attention_workspace_bytes() bytes for the
 *             same sizes, 256-byte aligned (may be NULL where that is 0).
 * The arithmetic: sums, maxima and lse are fp32.  Few rows a cache head: q as
 * whole numbers of 31 bits below its row's largest entry, a weight times its
 * value's scale as one of 30 bits below the largest of 64 tokens (with fp32
 * results, what that leaves too), products and their sums exact.  Many rows
 * (dtype bf16 or fp16): q as fp16 below 2^15 (entries below 2^-29 of the row's
 * largest lose bits), scores exact products summed in fp32, weights rounded to
 * fp16 for their product with the values (11 bits of those above 2^-21 of the
 * row's largest, none of those below 2^-32).
 * A NaN or an infinity in q makes that row NaN where it sees a position, and so
 * does a NaN key; a NaN value makes its 64 channels NaN in the rows that see it.
 */
size_t externd_kv4_attention_workspace_bytes(int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t dtype,
                                             int64_t tokens, int32_t batch, int32_t max_new, int64_t max_len);
/* Rows (new tokens x query heads of one cache head) that a workgroup of such a
 * call takes together: 4, the arithmetic of few rows above, or 256, that of
 * many rows; 0 on invalid arguments.                                        */
int32_t externd_kv4_attention_block_rows(int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t dtype,
                                         int64_t tokens, int32_t batch, int32_t max_new, int64_t max_len);
int externd_kv4_attention(const void* cache, int64_t num_pages, int32_t heads_kv, int32_t head_dim,
                          int32_t page_tokens, const void* q, int32_t dtype, int64_t q_token_stride,
                          int64_t q_head_stride, int32_t heads_q, void* out, float* lse, int64_t tokens,
                          int32_t batch, int32_t max_new, int64_t max_len, const int32_t* starts,
                          const int32_t* lens, const int32_t* table, int64_t table_pages, float scale,
                          int32_t window, void* workspace, size_t workspace_bytes, void* stream);

/* Log probabilities of given tokens: with z = scale x of each row,
 *   lse = ln sum_v exp z_v,  logprob = z_target - lse,
 *   entropy = lse - sum_v p_v z_v,  p = exp(z - lse),
 * and the `top` largest logits, the lower index first among equal ones (a NaN
 * with its sign clear counts above all): their indices and z - lse.
 *  logits     device, rows x vocab, row_stride >= vocab.
 *  targets    device int64[rows], or NULL with logprob NULL.  Below 0: no token
 *             is asked for, logprob 0.  vocab or more: logprob NaN.
 *  scale      finite, > 0 (1 / temperature).
 *  top        0 .. EXTERND_LOGPROBS_MAX_TOP, at most vocab; top_logprobs device
 *             fp32 and top_ids device int64, rows x top (NULL with top = 0).
 *  entropy, lse  device fp32[rows], each may be NULL.
 *  workspace  not used: externd_token_logprobs_workspace_bytes() is 0.
 * A row of nothing but -infinity: lse and log probabilities -infinity, entropy
 * 0.  A NaN or +infinity makes a row's lse, entropy and log probabilities NaN.
 * Sums are fp32 over at most 2^31 - 1 entries a row; rows < 2^26.           */
#define EXTERND_LOGPROBS_MAX_TOP 64
size_t externd_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t top);
int externd_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                           const int64_t* targets, float scale, int32_t top, float* logprob, float* entropy,
                           float* lse, float* top_logprobs, int64_t* top_ids, void* workspace,
                           size_t workspace_bytes, void* stream);

/* Gradient of the above for the logits:
 *   grad_v = scale [ g_logprob ([v = target] - p_v) - g_entropy p_v (ln p_v + entropy) ]
 * with the forward call's lse and entropy; g_logprob counts as 0 where a row
 * has no target.  Either gradient may be NULL (0); entropy may be NULL with
 * g_entropy.  grad: device, rows x vocab of dtype with its own row stride; it
 * may be `logits` itself with the same stride.  Where p_v = 0 its terms are 0,
 * in a row of nothing but -infinity too (the target's entry is scale g_logprob).
 * A target of vocab or more has no entry.                                   */
int externd_token_logprobs_backward(const void* logits, int32_t dtype, int64_t rows, int64_t vocab,
                                    int64_t row_stride, const int64_t* targets, float scale, const float* lse,
                                    const float* entropy, const float* g_logprob, const float* g_entropy,
                                    void* grad, int64_t grad_row_stride, void* stream);

/*
 * Operators at a model's dense ends, which its factorization leaves as they
 * are: the embedding, the head with the log probabilities behind it, and the
 * norm of all gradients.  The conventions of the decoding operators hold; the
 * innermost dimension of every array is dense, and outputs overlap no input
 * but where a call says so.
 */

/* Embedding: out[t] = scale table[ids[t]], rounded once; an id outside
 * [0, vocab) gives a row of zeros.
 *  table  device, vocab x width of dtype, table_stride >= width.
 *  ids    device int64[tokens]; out device, tokens x width, out_stride >= width.
 * vocab, width, tokens < 2^31; scale finite; tokens 0 is a valid call.       */
int externd_embedding(const void* table, int32_t dtype, int64_t vocab, int64_t width, int64_t table_stride,
                      const int64_t* ids, int64_t tokens, float scale, void* out, int64_t out_stride, void* stream);

/* Gradient of the above for the table:
 *   grad_table[v] = scale sum over the tokens t with ids[t] = v of grad[t],
 * summed in fp32 in an order that only ids and tokens decide and rounded once; ids outside [0, vocab)
 * add nothing, whatever grad holds there.  accumulate = 1: the sum is added
 * to what grad_table holds (the head's gradient, where the head is the
 * embedding), and rows without tokens are left as they are; 0: they become 0.
 *  workspace  device, >= externd_embedding_backward_workspace_bytes(), 256-byte
 *             aligned (may be NULL with tokens = 0).
 * tokens <= 2^26, vocab < 2^31 - 1, width <= 2^20.                           */
size_t externd_embedding_backward_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width);  /* 0 on invalid arguments */
int externd_embedding_backward(const void* grad, int32_t dtype, int64_t tokens, int64_t width, int64_t grad_stride,
                               const int64_t* ids, int64_t vocab, float scale, int32_t accumulate, void* grad_table,
                               int64_t grad_table_stride, void* workspace, size_t workspace_bytes, void* stream);

/* Log probabilities behind a dense head: externd_token_logprobs of the logits
 * x weight^T, which are never held.  With z = scale x weight^T, for each row
 *   lse = ln sum_v exp z_v,  logprob = z_target - lse,  entropy = lse - sum_v p_v z_v.
 *  x          device, rows x width of dtype, x_stride >= width; weight device,
 *             vocab x width of dtype, weight_stride >= width.
 *  targets    device int64[rows], or NULL with logprob NULL.  Below 0: no token
 *             is asked for, logprob 0.  vocab or more: logprob NaN.
 *  scale      finite, > 0.
 *  logprob, entropy, lse  device fp32[rows], each may be NULL.
 *  workspace  device, >= externd_linear_logprobs_workspace_bytes(), 256-byte aligned.
 * Logits are exact products summed in fp32 (fp32 operands enter as three bf16
 * parts each, whose products below 2^-24 of the largest are left out).  A logit
 * of -infinity counts as probability 0; a NaN or +infinity makes its row's
 * results NaN, and so do, in fp32, an infinity in x or weight.
 * rows <= 2^22, vocab <= 2^25, width <= 2^20, rows width <= 2^33, vocab width <= 2^37;
 * strides < 2^22.                                                           */
size_t externd_linear_logprobs_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t width);  /* 0 on invalid arguments */
int externd_linear_logprobs(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, int32_t dtype,
                            int64_t rows, int64_t vocab, int64_t width, const int64_t* targets, float scale,
                            float* logprob, float* entropy, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream);

/* Gradients of the above for x and weight: with the forward call's lse and
 * entropy and
 *   G_v = scale [ g_logprob ([v = target] - p_v) - g_entropy p_v (ln p_v + entropy) ],
 *   grad_x = G weight,  grad_weight = G^T x.
 * The logits are computed again, in pieces of the vocabulary.  g_logprob
 * counts as 0 where a row has no target (below 0, or vocab or more); either
 * gradient may be NULL (0), entropy may be NULL with g_entropy, and either
 * output may be NULL where it is not asked for.  A row whose two gradients are 0
 * takes no part, whatever x, lse and entropy hold there: its grad_x is 0.
 * rows = 0 gives a grad_weight of zeros.
 *  grad_x     device, rows x width of dtype; grad_weight device, vocab x width.
 *  workspace  device, >= externd_linear_logprobs_backward_workspace_bytes() with
 *             need_x, need_weight = whether the outputs are given; 256-byte aligned.
 * Sums are fp32; G enters its products in dtype (rounded to bf16, or to fp16
 * below 2^15 with a power of two for each row, the target's entry with what it
 * loses; an entry that p makes large keeps its half unit; fp32 as three bf16 parts).  In fp16 grad_weight takes x with such
 * powers as well: of all rows' largest |x| (|g_logprob| + |g_entropy| (1 + entropy)),
 * times scale, 2^-38 is left out of a row's part.                            */
size_t externd_linear_logprobs_backward_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t width,
                                                        int32_t need_x, int32_t need_weight);  /* 0 on invalid arguments */
int externd_linear_logprobs_backward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                                     int32_t dtype, int64_t rows, int64_t vocab, int64_t width, const int64_t* targets,
                                     float scale, const float* lse, const float* entropy, const float* g_logprob,
                                     const float* g_entropy, void* grad_x, int64_t grad_x_stride, void* grad_weight,
                                     int64_t grad_weight_stride, void* workspace, size_t workspace_bytes, void* stream);

/* The norm over many tensors, and clipping by it:
 *   norm = sqrt(sum over all entries of g^2),  out = g min(1, max_norm / norm).
 *  tensors    host array of `count` device pointers, each to sizes[i] dense
 *             entries of dtypes[i] (host arrays, not read after the call returns).
 *  out        host array of device pointers of the same sizes and types, each
 *             tensors[i] itself or apart from all tensors; NULL: in place.
 *  max_norm   >= 0; INFINITY: only the norm, and `out` is not written.
 *  norm       device fp32[1], out.
 *  workspace  device, >= externd_clip_gradients_workspace_bytes(count), 256-byte aligned.
 * The sum and the factor are fp64, so that no square overflows; a product is
 * rounded once after the factor's rounding to fp32.  A norm of 0 leaves all as
 * it is; an infinite one gives 0 (and NaN for infinite entries); NaN gives NaN.
 * count <= 2^20; sizes may be 0.  The same entry must not be in two tensors
 * that are written.                                                         */
size_t externd_clip_gradients_workspace_bytes(int64_t count);  /* 0 on invalid arguments */
int externd_clip_gradients(int64_t count, const void* const* tensors, void* const* out, const int64_t* sizes,
                           const int32_t* dtypes, double max_norm, float* norm, void* workspace,
                           size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* EXTERND_H */
