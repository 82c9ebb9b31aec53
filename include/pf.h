/*
 * pf.h -- C ABI of the low-rank pre-factorized layer library for NVIDIA B200 (sm_100a).
 *
 * The library computes the forward and backward passes of layers whose dense weight
 * W (k x n) has been replaced by two factors U (k x r) and V (n x r), W ~ U V^T
 * (Pufferfish, Section 2), plus the flat gradient buffer that is communicated once per
 * iteration (Section 4.1).
 *
 * Conventions common to every entry point
 *   - All tensor pointers are DEVICE pointers unless a parameter says "host".
 *   - The caller owns every buffer.  The library never allocates, frees or
 *     synchronises; all work is enqueued on `cuda_stream` (a cudaStream_t passed as
 *     void*, NULL = the legacy default stream) and returns immediately.
 *   - Inputs are never modified.  Outputs are overwritten (never accumulated into; where a call works in place or accumulates, it says so).
 *     No output may alias an input or another output.
 *   - All tensors of one call share `dtype`; products are accumulated in fp32 and
 *     rounded once (round-to-nearest-even) to `dtype` at the final store.  With
 *     PF_BF16 the on-chip intermediate x U (and dY V) is rounded to bf16 before the
 *     second product.
 *   - Matrices are row-major.  A leading dimension `ld*` is the distance in ELEMENTS
 *     between consecutive rows and must be >= the row length.
 *   - `workspace` is caller-provided scratch of at least the matching
 *     pf_*_workspace() query, 256-byte aligned; its contents are undefined afterwards.
 *     Two calls that may overlap on the GPU must not share a workspace.
 *   - Besides the workspace the library keeps a few fixed device arrays of its own (a
 *     status word and 40 KB of counters at which the thread blocks of a split reduction
 *     meet).  A reduction over the batch (dU, dV, and x U / dY V when the batch is small) is
 *     cut into slices whose thread blocks wait for one another inside one launch, so all
 *     of them must be resident at once: the library sizes such a launch to at most one block
 *     per SM of the device, which guarantees that on an otherwise idle GPU.  Kernels of
 *     other streams (or processes) that occupy SMs at the same time can delay a sibling
 *     block; the wait is bounded (about two seconds), after which the launch gives up, leaves
 *     its outputs unwritten and pf_last_device_status() reports PF_ERR_TIMEOUT.  Calls of this
 *     library on different streams of equal priority may be in flight together (each launch
 *     takes the next of 32 counter sets: keep at most 32 such calls unfinished per device);
 *     do not mix stream priorities, and do not run backward calls beside long-running
 *     kernels that pin most SMs.
 *   - Gradients that are sums over the batch (dU, dV) are added in a fixed order:
 *     repeating a call on the same inputs gives bit-identical results.
 *   - Every entry returns a pf_status.  Errors detected on the host (bad pointer,
 *     bad dimension, workspace too small, ...) are returned BEFORE anything is
 *     launched.  Nothing is printed, nothing aborts.
 *   - Problems with no rows / no tensors (m = 0, N = 0, count = 0) are PF_OK no-ops.
 */
#ifndef PF_H_
#define PF_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PF_OK = 0,
    PF_ERR_INVALID_ARG = 1, /* null required pointer, dimension < 1, ld too small, bad dtype,
                               misaligned pointer, negative count */
    PF_ERR_UNSUPPORTED = 2, /* valid mathematics outside the implemented envelope */
    PF_ERR_WORKSPACE = 3,   /* workspace missing, misaligned or too small; pack capacity too small */
    PF_ERR_CUDA = 4,        /* a CUDA runtime / driver call or a launch failed */
    PF_ERR_TIMEOUT = 5      /* a bounded device-side wait expired (see pf_last_device_status) */
} pf_status;

typedef enum {
    PF_F32 = 0, /* fp32 storage and accuracy: tensor-core products of exactly split operands (three bf16 parts, fp32
                   accumulation), fp32 FMA arithmetic where a layout does not allow them.  Subnormal operands count in
                   full.  Outputs that an infinity, a NaN, an operand from 2^112 on or a sum from 2^96 on reaches are
                   computed again with FMAs, with the whole tile around them, and are what FMA arithmetic gives. */
    PF_BF16 = 1 /* bf16 storage, tensor-core products with fp32 accumulation */
} pf_dtype;

/* Static, human-readable name of a status code. */
const char* pf_status_string(int status);

/* Library version, major*10000 + minor*100 + patch. */
int pf_version(void);

/* Number of kernels this library has launched in this process so far (monotonic, all
 * devices and streams).  Lets a caller verify that work ran in this library's kernels. */
long long pf_launch_count(void);

/* Device-side status of the current device: PF_OK, or PF_ERR_TIMEOUT if a kernel of
 * this library gave up on a bounded wait since the last query.  Synchronises the
 * device (blocking) and clears the flag.  Never needed on the normal path. */
int pf_last_device_status(void);

/* ---------------------------------------------------------------------------------
 * Factorized fully-connected layer   y = (x U) V^T
 * (Section 2.1 "Low-rank factorization for FC layers"; Appendix B "FC layer", whose
 *  row convention (xU)V^T is used: U is the input-side factor, V the output-side one.)
 *
 *   x [m, k] (ldx)   U [k, r] (ldu)   V [n, r] (ldv)   y [m, n] (ldy)
 *   T_stash [m, r] (ldt): optional output, the intermediate T = x U rounded to `dtype`,
 *                         for reuse by the backward pass; NULL = not written.
 * m >= 0; k, n, r >= 1 (r need not divide anything; r > min(k, n) is legal).
 * ------------------------------------------------------------------------------- */
size_t pf_lowrank_linear_workspace(int64_t m, int64_t k, int64_t n, int64_t r,
                                   int dtype, int is_bwd);

int pf_lowrank_linear_fwd(const void* x, int64_t ldx, const void* U, int64_t ldu,
                          const void* V, int64_t ldv, void* y, int64_t ldy,
                          void* T_stash, int64_t ldt,
                          int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                          void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The forward with the bias and activation that follow the layer in a network:
 *   y = act((x U) V^T + bias)
 * the first half of the factorized feed-forward block FFN(x) = max(0, x W1 + b1) W2 + b2 with
 * W1 = U1 V1^T (Section 2.4; biases are not factorized, Section 2.1), or, with PF_ACT_NONE, any
 * factorized layer followed by its bias (the second half of the FFN, the LSTM gate pre-activations
 * of Section 2.3).
 *   bias [n] in `dtype`, contiguous; NULL = no bias.     act: PF_ACT_NONE or PF_ACT_RELU.
 * bias and activation are applied to the fp32 result before the single rounding to `dtype` (PF_BF16 layouts
 * that only the FMA kernels take: y is stored first and a second pass applies them in place, two roundings).
 * T_stash is x U as in pf_lowrank_linear_fwd (bias does not enter it).
 * Same workspace, pitches and error behaviour as pf_lowrank_linear_fwd; an act outside the enum is
 * PF_ERR_INVALID_ARG.  The backward of the activation (dY masked by y > 0) and the bias gradient
 * (column sums of dY) are the caller's: pf_lowrank_linear_bwd takes the gradient of (x U) V^T. */
typedef enum {
    PF_ACT_NONE = 0,
    PF_ACT_RELU = 1 /* max(0, .) */
} pf_act;
int pf_lowrank_linear_fwd_act(const void* x, int64_t ldx, const void* U, int64_t ldu,
                              const void* V, int64_t ldv, const void* bias, int act,
                              void* y, int64_t ldy, void* T_stash, int64_t ldt,
                              int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                              void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The step of the backward pass that undoes pf_lowrank_linear_fwd_act's epilogue, before
 * pf_lowrank_linear_bwd is called with the result: for y = act(z + bias) and an upstream dY [m, n],
 *   dZ   = dY where y > 0, 0 elsewhere (PF_ACT_RELU);  dZ = dY (PF_ACT_NONE)     written OVER dY
 *   dbias[j] = sum over the m rows of dZ[:, j]  (plain sum, fp32 accumulation in a fixed order,
 *              rounded once to `dtype`)                    [n], NULL = not wanted
 * (Section 2.4: the feed-forward block max(0, x W1 + b1) W2 + b2; biases are trained unfactorized,
 * Section 2.1.)  y (ldy) is the forward's output and is read only for PF_ACT_RELU.  The workspace of
 * pf_bias_act_bwd_workspace(m, n) bytes is needed only when dbias is given.  One launch, two
 * with dbias and more than 4096 rows; m = 0 zeroes dbias. */
size_t pf_bias_act_bwd_workspace(int64_t m, int64_t n);
int pf_bias_act_bwd(const void* y, int64_t ldy, void* dY, int64_t lddy, void* dbias,
                    int64_t m, int64_t n, int act, int dtype,
                    void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The same forward for callers that cannot allocate device memory and therefore have no
 * workspace to pass: latency-critical host paths where cudaMalloc is forbidden because it
 * synchronises the device, plug-ins that are handed tensors but no allocator, and processes
 * whose device memory is already fully committed to a pool they do not control.
 * (The paper has no counterpart; this is a deployment variant.)
 *
 * Identical to pf_lowrank_linear_fwd except that the scratch is a fixed array inside the
 * library image (PF_STATIC_SCRATCH_BYTES per GPU that loads the library, held until the
 * process exits).  It calls no cudaMalloc / cudaFree and no allocating library routine.
 *   - The bound is the scratch this call will really use, which depends on the path its
 *     sizes, pointers and pitches select (it can be far below the public workspace query, which
 *     reserves for every path): many rows at a small rank (m >= 2048, r <= 192, 16-byte aligned
 *     rows) take the fused kernel, which keeps x U on chip and needs nothing when the stash
 *     is written directly; otherwise one m x r copy of x U, the fp32 slices of a split first
 *     product, and re-pitched copies of operands whose row pitch is not a multiple of 16 bytes.
 *     Only where the fused kernel would need nothing but cannot store rows of y or of the stash
 *     (a width that is no multiple of 8 at a 16-byte pitch), as many rows at a time as fit.
 *     A call that needs more than PF_STATIC_SCRATCH_BYTES is rejected with PF_ERR_WORKSPACE
 *     before anything is launched.  Of the benchmark shapes both Transformer-FFN layers fit,
 *     the LSTM gate layer (700 x 1500 -> 6000, r = 375) fits with 16-byte row pitches and is
 *     refused with its tight 3000 / 750-byte pitches.
 *   - The first call on each device is the set-up call: it looks up the array's device address
 *     with that device current, and (the driver loads modules lazily) it is also when the array
 *     itself is materialised, so free device memory drops once, by the array's size; no later
 *     call changes it.  Make that first call outside any stream capture.
 *   - All calls on a device share the one array, which keeps whatever the previous call
 *     left in it: two calls that may overlap on the GPU (different streams) race and must be
 *     ordered by the caller.  Nothing in the array has to be cleared between calls.
 * pf_static_scratch_bytes() returns PF_STATIC_SCRATCH_BYTES as compiled. */
#define PF_STATIC_SCRATCH_BYTES (8u << 20)
int pf_lowrank_linear_fwd_static(const void* x, int64_t ldx, const void* U, int64_t ldu,
                                 const void* V, int64_t ldv, void* y, int64_t ldy,
                                 void* T_stash, int64_t ldt,
                                 int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                                 void* cuda_stream);
size_t pf_static_scratch_bytes(void);

/* Gradients of the layer above for an upstream gradient dY [m, n] (chain rule on
 * y = (xU)V^T; plain sums over the m rows, no averaging):
 *   G  = dY V           [m, r]  (kept on chip / in workspace)
 *   dX = G U^T          [m, k]  (lddx)   NULL = not wanted (first layer)
 *   dU = x^T G          [k, r]  (lddu)
 *   dV = dY^T (x U)     [n, r]  (lddv)
 * T_stash [m, r] (ldt): the forward's stashed x U, or NULL to have it recomputed. */
int pf_lowrank_linear_bwd(const void* x, int64_t ldx, const void* U, int64_t ldu,
                          const void* V, int64_t ldv, const void* dY, int64_t lddy,
                          const void* T_stash, int64_t ldt,
                          void* dX, int64_t lddx, void* dU, int64_t lddu, void* dV, int64_t lddv,
                          int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                          void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The same backward with two options for the factor gradients, as gradient accumulation over
 * micro-batches and fp32 master gradients need them (the paper trains with mixed precision and
 * all-reduces the factor gradients, Sections 4.1 and 3; it does not spell these variants out):
 *   PF_GRAD_ACCUMULATE  dU and dV are ADDED to what the matrices hold: dU <- dU + x^T G, dV <- dV + dY^T (xU)
 *                       (the caller zeroes them before the first micro-batch);
 *   PF_GRAD_F32         dU [k, r] and dV [n, r] are fp32 matrices (lddu, lddv in floats) whatever
 *                       `dtype` is: with PF_BF16 the fp32 sums are stored unrounded.
 * dX is never accumulated and stays in `dtype`.  flags = 0 is pf_lowrank_linear_bwd.  The call runs
 * the same kernels as the plain backward, with the plain gradients directed into the workspace, and
 * one more small launch writes the caller's matrices: where a reduction over the batch left its fp32 slices in the
 * workspace (split ones, every benchmark shape among them, and whole ones unless the tiles of dU and dV are more than
 * the SMs) from those, summed again in the same order, so that the values are the unrounded fp32 sums (rounded
 * once when added into a PF_BF16 matrix); on the remaining paths from the plain gradient (PF_BF16: the
 * micro-batch's gradient has then been rounded to bf16 before it is widened or added).  With PF_BF16 the sums are those of
 * the tensor cores (relative error 1e-7 to 5e-6, growing with the rows of a slice) of operands T and G that were
 * rounded to bf16, which weighs about 1.7e-3.
 * Same workspace query, pitches and errors as pf_lowrank_linear_bwd; unknown flag bits are
 * PF_ERR_INVALID_ARG.  With m = 0 and PF_GRAD_ACCUMULATE nothing is written. */
#define PF_GRAD_ACCUMULATE 1u
#define PF_GRAD_F32 2u
int pf_lowrank_linear_bwd_ex(const void* x, int64_t ldx, const void* U, int64_t ldu,
                             const void* V, int64_t ldv, const void* dY, int64_t lddy,
                             const void* T_stash, int64_t ldt,
                             void* dX, int64_t lddx, void* dU, int64_t lddu, void* dV, int64_t lddv,
                             int64_t m, int64_t k, int64_t n, int64_t r, int dtype, unsigned flags,
                             void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Grouped factorized fully-connected layers: `groups` layers of ONE shape (m, k, n, r), each with its
 * own factor pair (U_g, V_g), in one call -- the per-gate factorization of an LSTM layer
 * (Section 2.3, eq. "lr-lstm-rule": every gate matrix W_i*, W_h* is replaced by its own U V^T; the
 * LSTM table of the appendix lists the 1500 x 375 / 375 x 1500 factors per gate) and the four
 * projections W^Q, W^K, W^V, W^O of a factorized attention block (Section 2.4).
 *     y_g = (x_g U_g) V_g^T ,   g = 0 .. groups-1
 * Every tensor of group g starts s* ELEMENTS after that of group g-1 (sx for x, su for U, ...); the
 * matrices themselves are as in the ungrouped calls.  sx = 0 means ONE input x shared by all groups
 * (the gates of an LSTM all read the same x_t); factors and outputs are always per group.
 * With bf16 and 16-byte aligned pointers, pitches and strides the whole call is two launches
 * (all x_g U_g, then all T_g V_g^T, or half of the groups each), whatever `groups`; ragged widths (not a multiple of 8) add one launch
 * that copies those operands to 16-byte pitches; other layouts, and fp32, run group by group through the
 * ungrouped kernels (same results, more launches).
 *
 * Backward, for dY_g [m, n] (stride sdy):
 *   dU_g = x_g^T (dY_g V_g),  dV_g = dY_g^T (x_g U_g)                       (strides sdu, sdv)
 *   dX_g = (dY_g V_g) U_g^T   (stride sdx)            when every group has its own x (sx != 0);
 *   dX   = sum over g of (dY_g V_g) U_g^T, ONE m x k matrix (sdx ignored)   when x is shared (sx = 0),
 *          since a shared input collects the gradient of every group that reads it.
 *   NULL dX = not wanted.  T_stash (stride st): the forward's stash, or NULL to recompute.
 * Two launches (three when T is recomputed) on the fast path, one more for ragged widths.
 * ------------------------------------------------------------------------------- */
size_t pf_lowrank_linear_grouped_workspace(int groups, int64_t m, int64_t k, int64_t n, int64_t r,
                                           int dtype, int is_bwd);

int pf_lowrank_linear_grouped_fwd(int groups,
                                  const void* x, int64_t ldx, int64_t sx,
                                  const void* U, int64_t ldu, int64_t su,
                                  const void* V, int64_t ldv, int64_t sv,
                                  void* y, int64_t ldy, int64_t sy,
                                  void* T_stash, int64_t ldt, int64_t st,
                                  int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream);

int pf_lowrank_linear_grouped_bwd(int groups,
                                  const void* x, int64_t ldx, int64_t sx,
                                  const void* U, int64_t ldu, int64_t su,
                                  const void* V, int64_t ldv, int64_t sv,
                                  const void* dY, int64_t lddy, int64_t sdy,
                                  const void* T_stash, int64_t ldt, int64_t st,
                                  void* dX, int64_t lddx, int64_t sdx,
                                  void* dU, int64_t lddu, int64_t sdu,
                                  void* dV, int64_t lddv, int64_t sdv,
                                  int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Factorized convolution: a kh x kw convolution into R channels (factor U) followed by a
 * 1 x 1 convolution to O channels (factor V), nothing in between
 * (Section 2.2 "Factorizing a convolution layer"; Appendix B "Convolution layer").
 * Cross-correlation (no kernel flip), zero padding `pad`, stride `stride` on the
 * kh x kw convolution only; no dilation, no groups.
 *
 *   x [N, H, W, C] NHWC, contiguous
 *   U [kh, kw, C, R]  = the unrolled (kh*kw*C) x R matrix of Section 2.2, rows tap-major
 *   V [O, R]
 *   y [N, Ho, Wo, O] NHWC,  Ho = (H + 2 pad - kh) / stride + 1 (floor), Wo likewise
 *   T_stash [N, Ho, Wo, R]: optional output of the thin convolution; NULL = not written.
 * Returns PF_ERR_UNSUPPORTED for kh != kw or stride < 1.
 * bf16: the query is what the fastest kernels use.  A smaller workspace is taken down to what the slower ones cannot do without
 * (T; backwards also dT, both of R elements per pixel, and the sums of the reductions), and selects those.
 * ------------------------------------------------------------------------------- */
size_t pf_lowrank_conv_workspace(int N, int H, int W, int C, int R, int O,
                                 int kh, int kw, int stride, int pad, int dtype, int is_bwd);

int pf_lowrank_conv_fwd(const void* x, const void* U, const void* V, void* y, void* T_stash,
                        int N, int H, int W, int C, int R, int O,
                        int kh, int kw, int stride, int pad, int dtype,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Gradients of the factorized convolution for dY [N, Ho, Wo, O]:
 *   dT = dY V (per pixel), dV [O, R] = dY^T T, dU [kh, kw, C, R] = im2col(x)^T dT,
 *   dX [N, H, W, C] = transposed convolution of dT with U (NULL = not wanted).
 * T_stash: the forward's stash or NULL to recompute. */
int pf_lowrank_conv_bwd(const void* x, const void* U, const void* V, const void* dY,
                        const void* T_stash, void* dX, void* dU, void* dV,
                        int N, int H, int W, int C, int R, int O,
                        int kh, int kw, int stride, int pad, int dtype,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);

/* pf_lowrank_conv_bwd with the gradient options of pf_lowrank_linear_bwd_ex (PF_GRAD_ACCUMULATE,
 * PF_GRAD_F32) for dU [kh, kw, C, R] and dV [O, R]; same mechanism (or, where the launches of the backward
 * add up their slices themselves, no launch more: the same sums), same workspace query. */
int pf_lowrank_conv_bwd_ex(const void* x, const void* U, const void* V, const void* dY,
                           const void* T_stash, void* dX, void* dU, void* dV,
                           int N, int H, int W, int C, int R, int O, int kh, int kw, int stride,
                           int pad, int dtype, unsigned flags, void* workspace, size_t workspace_bytes,
                           void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Flat gradient buffer (Section 4.1 "Implementation details and optimizations": all
 * gradient tensors are packed into one flat buffer so that one all-reduce per iteration
 * suffices).  Copies tensor i (numels[i] elements of `dtype`) bit for bit to
 * flat[offsets_out[i] ...], in list order, tightly (no padding, no conversion, no scaling):
 *   offsets_out[0] = 0, offsets_out[i+1] = offsets_out[i] + numels[i].
 *
 *   grads        host array of `count` device pointers (element-aligned)
 *   numels       host array of `count` element counts (>= 0)
 *   flat         device buffer of `flat_capacity_elems` elements
 *   offsets_out  host array of count+1 entries, written before return (element units)
 * No workspace is needed (workspace arguments are accepted and ignored).
 * PF_ERR_WORKSPACE if the tensors do not fit in flat_capacity_elems.
 * ------------------------------------------------------------------------------- */
int pf_pack_factor_grads(const void* const* grads, const int64_t* numels, int count, int dtype,
                         void* flat, int64_t flat_capacity_elems, int64_t* offsets_out,
                         void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The inverse of pf_pack_factor_grads, for the step after the all-reduce of the flat buffer
 * (Section 4.1: one buffer is communicated per iteration; every factor then needs its own averaged
 * gradient back): tensor i receives flat[offsets_out[i] .. offsets_out[i] + numels[i]) bit for bit,
 * with the same tight offsets (prefix sums of numels, written to offsets_out before return).
 *   flat   device buffer of `flat_elems` elements (read only)
 *   grads  host array of `count` device pointers (element-aligned), the destinations
 * PF_ERR_WORKSPACE if the list is longer than flat_elems.  No workspace is needed. */
int pf_unpack_factor_grads(const void* flat, int64_t flat_elems, void* const* grads, const int64_t* numels,
                           int count, int dtype, int64_t* offsets_out,
                           void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Tokens of a layer with experts, for the grouped layers above: [experts, capacity, k] is the grouped forward's x with one
 * factor pair per expert.  `tokens` tokens choose `k` of `experts` experts each; assignment a = token * k + j goes to
 * expert ids[a].  (The paper has no counterpart; a factorized feed-forward layer is the expert.)
 *
 * pf_expert_sort gives every assignment a row.  An expert's assignments keep their order; the r-th of expert e gets row
 *   capacity > 0:  e * capacity + r, none from r = capacity on;      rows = experts * capacity
 *   capacity = 0:  offsets[e] + r, expert after expert without gaps;  rows = tokens * k
 * An id outside 0 .. experts - 1 gets no row.  The same expert may be chosen twice by a token (two rows).
 *   ids     [tokens, k]   int32
 *   slots   [tokens, k]   int32  row of each assignment, -1 for none
 *   sources [rows]        int32  assignment of each row, -1 for none
 *   counts  [experts]     int32  assignments that chose the expert, those without a row among them
 *   offsets [experts + 1] int32  first row of each expert; behind the last, experts * capacity or the rows in use
 * One launch and no workspace up to 32768 assignments; two launches and pf_expert_sort_workspace bytes beyond.  PF_ERR_UNSUPPORTED: more than
 * 2048 experts, or 2^30 assignments or rows.
 * pf_expert_rows returns `rows` (0 for sizes that pf_expert_sort refuses).
 *
 * The other four take slots and sources as pf_expert_sort left them (an index outside the rows counts as none) and
 * matrices of `width` columns at any pitch; x, y, dx, dy have `tokens` rows, xs, ys, dxs, dys `rows`:
 *   dispatch_fwd   xs[slots[t, j]] = x[t]; rows without an assignment are zeroed
 *   dispatch_bwd   dx[t]  = sum over j of dxs[slots[t, j]]
 *   combine_fwd    y[t]   = sum over j of weights[t, j] ys[slots[t, j]]                weights [tokens, k] fp32, NULL = ones
 *   combine_bwd    dys[slots[t, j]] = weights[t, j] dy[t], other rows zeroed;  dweights[t, j] = <dy[t], ys[slots[t, j]]>, 0 without a row
 *                  (dys or dweights may be NULL: not wanted; weights may not: the gradient of a sum without weights is dispatch_fwd of dy)
 * Sums run over j in order, in fp32, and are rounded once; assignments without a row add nothing, so a token all of whose
 * assignments were dropped gives zeros.  dweights is fp32.  What rows without an assignment hold is never read.  (PF_BF16 rows with an odd start,
 * width or pitch are read in aligned 4-byte words, so that two bytes beside a row may be read; they are not used.)  One launch each, no workspace.
 *
 * The grouped layers take rows with a capacity: their groups have one shape.  Rows without gaps are for a caller's own products over
 * offsets[e] .. offsets[e + 1].
 * ------------------------------------------------------------------------------- */
int64_t pf_expert_rows(int64_t tokens, int k, int experts, int64_t capacity);

size_t pf_expert_sort_workspace(int64_t tokens, int k, int experts);

int pf_expert_sort(const int32_t* ids, int64_t tokens, int k, int experts, int64_t capacity,
                   int32_t* slots, int32_t* sources, int32_t* counts, int32_t* offsets,
                   void* workspace, size_t workspace_bytes, void* cuda_stream);

int pf_expert_dispatch_fwd(const void* x, int64_t ldx, const int32_t* slots, const int32_t* sources, void* xs, int64_t ldxs,
                           int64_t tokens, int k, int64_t rows, int64_t width, int dtype, void* cuda_stream);

int pf_expert_dispatch_bwd(const void* dxs, int64_t lddxs, const int32_t* slots, void* dx, int64_t lddx,
                           int64_t tokens, int k, int64_t rows, int64_t width, int dtype, void* cuda_stream);

int pf_expert_combine_fwd(const void* ys, int64_t ldys, const int32_t* slots, const float* weights, void* y, int64_t ldy,
                          int64_t tokens, int k, int64_t rows, int64_t width, int dtype, void* cuda_stream);

int pf_expert_combine_bwd(const void* ys, int64_t ldys, const int32_t* slots, const int32_t* sources, const float* weights,
                          const void* dy, int64_t lddy, void* dys, int64_t lddys, float* dweights,
                          int64_t tokens, int k, int64_t rows, int64_t width, int dtype, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Norm and position rotation of queries and keys, for each head: what follows the projections W^Q and W^K of an attention
 * layer (Section 2.4; grouped layers above) where its heads are normalised and its positions are rotations.  For a row x of
 * `dim` elements (one head of the token at position t):
 *   z = x / sqrt(mean(x^2) + eps) * w,   then the first rot_dim elements of z are pairs (a, b), pair i turned by t * inv_freq[i]:
 *   (a, b) -> (a cos - b sin, b cos + a sin)
 * PF_ROPE_HALVES pairs element i with rot_dim / 2 + i, PF_ROPE_PAIRS element 2 i with 2 i + 1; the other elements stay as they are.
 *   q, q_out [tokens, q_heads, dim]: token t's head h starts at t * ldq + h * sq ELEMENTS; k, k_out likewise (k_heads).  Any
 *            strides under which rows do not overlap (heads inside tokens or tokens inside heads); elements of a row are contiguous.
 *   wq, wk   [dim] in `dtype`, NULL = ones        inv_freq [rot_dim / 2] fp32 (below 2^31; one that is not finite makes its pair NaN)
 *   positions [tokens] int64, NULL = 0, 1, 2, ...
 * Statistics and products are in fp32 and rounded once.  An angle is counted in parts of a turn, those of one position rounded to
 * 2^-65 of a turn (2^-64 for frequencies above 2^20), so that far positions (up to 2^40: off by 2^-25 of a turn there) keep it; sine and cosine of it to fp32 (to
 * 2^-20 with PF_BF16).  Either of q_heads and k_heads may be 0 (its pointers are ignored then).  rot_dim is even,
 * 0 .. dim.  (Of PF_BF16 rows and weights that do not start and end on 4 bytes, two bytes beside them may be read; they are not used.)
 * PF_ERR_UNSUPPORTED: dim > 1024, more than 65536 heads or 2^30 tokens.  One launch, no workspace.
 *
 * Backward, for the gradients dq_out and dk_out of the outputs: dq, dk (in `dtype`; always written), and dwq, dwk [dim] (sums over
 * tokens and heads in a fixed order, fp32, rounded once; NULL = not wanted).  The norm's statistics are computed again from q and k.
 * flags: PF_GRAD_ACCUMULATE adds to dwq and dwk (dq and dk are never accumulated), PF_GRAD_F32 makes them fp32.  The workspace is
 * needed only when dwq or dwk is given, which also takes a second launch.  tokens = 0 zeroes dwq and dwk (accumulating: leaves them).
 * ------------------------------------------------------------------------------- */
typedef enum {
    PF_ROPE_HALVES = 0,
    PF_ROPE_PAIRS = 1
} pf_rope_style;

int pf_qk_norm_rope_fwd(const void* q, int64_t ldq, int64_t sq, const void* k, int64_t ldk, int64_t sk,
                        const void* wq, const void* wk, const int64_t* positions, const float* inv_freq,
                        void* q_out, int64_t ldqo, int64_t sqo, void* k_out, int64_t ldko, int64_t sko,
                        int64_t tokens, int q_heads, int k_heads, int dim, int rot_dim, int style, double eps, int dtype,
                        void* cuda_stream);

size_t pf_qk_norm_rope_bwd_workspace(int64_t tokens, int q_heads, int k_heads, int dim);

int pf_qk_norm_rope_bwd(const void* q, int64_t ldq, int64_t sq, const void* k, int64_t ldk, int64_t sk,
                        const void* wq, const void* wk, const int64_t* positions, const float* inv_freq,
                        const void* dq_out, int64_t lddqo, int64_t sdqo, const void* dk_out, int64_t lddko, int64_t sdko,
                        void* dq, int64_t lddq, int64_t sdq, void* dk, int64_t lddk, int64_t sdk, void* dwq, void* dwk,
                        int64_t tokens, int q_heads, int k_heads, int dim, int rot_dim, int style, double eps, int dtype,
                        unsigned flags, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * AdamW over a list of tensors, IN PLACE: the step behind the exchange of the flat gradient buffer (Section 4.1).  Tensor i of
 * numels[i] elements, t = step:
 *   g = grad_scale * grad        m <- beta1 m + (1 - beta1) g        v <- beta2 v + (1 - beta2) g^2
 *   p <- p - lr (weight_decay p + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps))
 * in fp32, m and v with each product and sum rounded by itself; eps sqrt(1 - beta2^t) below 2^-63
 * counts as 2^-63.
 *   params   in param_dtype.  masters: NULL, or (PF_BF16 parameters) fp32 masters, which are then what is read and stepped;
 *            params receives them rounded.  Without masters a PF_BF16 parameter is stepped in fp32 and rounded once.
 *   grads    in grad_dtype, read only: the slices of a flat buffer as they are (element alignment) or any other tensors
 *   state    PF_STATE_F32: m, v fp32.
 *            PF_STATE_8BIT: m is 8-bit floats of the e4m3 format, v of the e5m2 format, each times the fp32 scale of its block of 256
 *            elements (counted from the tensor's first): m_scales, v_scales [ceil(numels[i] / 256)].  Zeroed codes and scales are
 *            the state before the first step.  Scales are powers of two that put the largest of a block into [128, 256) (m) and [2^14, 2^15) (v).
 *            A value is rounded up with the probability of what is cut off (16 bits of a hash of seed, i and the element's place in its
 *            tensor; give each step another seed): rounding to nearest would leave v as it is once 1 - beta2 is
 *            below half a step of the format.  Under the format's smallest normal number m becomes 0 and v > 0 that number, so that a block's
 *            smallest elements hardly move: with betas 0.9 and 0.98 and steady gradients of 2^-12 to 2^-13 of the block's largest the mean update is two
 *            thirds of AdamW's, below that a tenth, below 2^-16 a fiftieth; down to 2^-12 it is AdamW's (1.01 of it).  What is not
 *            finite becomes NaN.  p is stepped with m and v before they are rounded.
 * numels, and the lists of pointers, are host arrays of `count`; tensors with numels 0 are skipped (but count as places).  The
 * arrays of different tensors must not overlap.
 * scalars: NULL, or a device array (4-byte aligned) that replaces lr, step (by the two corrections), grad_scale and seed, for
 * steps replayed from a CUDA graph.  The library reads it when the step runs.
 * One launch for up to 448 tensors, no workspace. */
typedef enum {
    PF_STATE_F32 = 0,
    PF_STATE_8BIT = 1
} pf_state;
typedef struct {
    double lr, beta1, beta2, eps, weight_decay; /* finite; 0 <= beta < 1, eps >= 0 */
    int64_t step;                               /* t >= 1: 1 for the first step */
    float grad_scale;                           /* 1 = none; the inverse of a loss scale, a clipping factor */
    uint32_t seed;                              /* of the rounding of 8-bit states */
} pf_adamw;
typedef struct {
    float lr;
    float correction1, correction2; /* 1 - beta1^t, 1 - beta2^t */
    float grad_scale;
    uint32_t seed;
} pf_adamw_scalars;
int pf_adamw_step(void* const* params, float* const* masters, const void* const* grads, void* const* m, void* const* v,
                  float* const* m_scales, float* const* v_scales, const int64_t* numels, int count,
                  int param_dtype, int grad_dtype, int state, const pf_adamw* hyper, const pf_adamw_scalars* scalars,
                  void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * A residual's addition and the root-mean-square norm that follows, in front of a block's layers (Section 2.4).  For each of `tokens` rows:
 *   h = x + residual (residual NULL: h = x)          y = h / sqrt(mean(h^2) + eps) * w
 *   w [width] in `dtype`, NULL = ones.   h and y in `dtype`; y is made of the unrounded sum.
 *   y8, scales: y in 8 bits as well, or instead: codes are 8-bit floats of the e4m3 format (a byte each, ldy8 in bytes), each times the fp32 scale of its block
 *            of `block` elements (32 or 128, counted from the row's first; 0: the whole row).  A scale is 1 / 448 of the largest of
 *            its block (2^-126 at least; 0 for a block of zeros), so codes reach 448; a value is rounded once, to nearest.  scales [tokens, ceil(width / block)],
 *            contiguous.
 * Each of h, y and (y8, scales) may be NULL: not wanted; not all of them.  h may be residual or x (in place), with its pitch.
 * A row whose h holds an infinity or a NaN gives NaN in every element (codes and scales as well; backward: dx).  Statistics and products are in fp32, of rows scaled by a
 * power of two where their squares would leave its range.
 * PF_ERR_UNSUPPORTED: width > 16384.  One launch, no workspace.
 *
 * Backward, for the gradient dy of y and, NULL = none, dh of h (what reaches the sum by the residual's way):
 *   dx = dh + the gradient of the norm at h: that of x and of the residual alike;    dw [width] = sum over rows (fixed order, fp32, rounded once)
 * h is the forward's (rounded); its statistics are computed again.  dx may be dh, dy or h, with its pitch.  dw NULL = not wanted.  flags: PF_GRAD_ACCUMULATE
 * adds to dw, PF_GRAD_F32 makes it fp32.  The workspace is needed only with dw, which also takes a second launch.  tokens = 0 zeroes dw (accumulating: leaves it).
 * (Of PF_BF16 rows that do not start and end on 4 bytes, two bytes beside them may be read; they are not used.)
 * ------------------------------------------------------------------------------- */
int pf_add_rms_norm_fwd(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* w, void* h, int64_t ldh,
                        void* y, int64_t ldy, void* y8, int64_t ldy8, float* scales, int block,
                        int64_t tokens, int64_t width, double eps, int dtype, void* cuda_stream);

size_t pf_add_rms_norm_bwd_workspace(int64_t tokens, int64_t width);

int pf_add_rms_norm_bwd(const void* h, int64_t ldh, const void* w, const void* dy, int64_t lddy, const void* dh, int64_t lddh,
                        void* dx, int64_t lddx, void* dw, int64_t tokens, int64_t width, double eps, int dtype, unsigned flags,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Gated factorized layers: two factor pairs of one shape that read one x, as two groups of the grouped layers above (su, sv, st: elements between the
 * matrices of the pairs), and the product of one's activation with the other:
 *   g = (x U0) V0^T + bias0        u = (x U1) V1^T + bias1        y = act(g) * u            y [m, n]
 *   bias [2, n] in `dtype`, contiguous; NULL = none.     act: a pf_gate.
 *   T_stash [2, m, r]: as in the grouped forward; NULL = not written.
 * With PF_BF16 x U is rounded to bf16 before the second product, as everywhere; g and u stay in fp32 up to the one rounding of y.  (k or n above 2^22: g and u
 * are rounded as well.)
 * Two launches, one more where matrices at a base, pitch or stride that is not a multiple of 16 bytes are copied (x of k a multiple of 8: two for each 2^23 of its elements); fp32: both pairs' products side by side and one launch for the gate, for some rows at a time; the smallest fp32 layers and
 * other layouts: the launches of the grouped layer and one for the gate.
 *
 * Backward, for dY [m, n]: g and u are computed again,
 *   dZ0 = dY * u * act'(g),  dZ1 = dY * act(g)    (rounded to `dtype`; act' of max(0, .) is 0 at 0)
 * and from them what the grouped backward with a shared x gives: dX [m, k] (NULL = not wanted), dU [2, k, r] (sdu), dV [2, n, r] (sdv), and
 * dbias [2, n] (NULL = not wanted).  T_stash: the forward's, or NULL to have it recomputed.
 * ------------------------------------------------------------------------------- */
typedef enum {
    PF_GATE_SILU = 0,    /* g / (1 + e^-g) */
    PF_GATE_GELU = 1,    /* g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2 */
    PF_GATE_SIGMOID = 2, /* 1 / (1 + e^-g) */
    PF_GATE_RELU = 3     /* max(0, g) */
} pf_gate;

size_t pf_lowrank_linear_gated_workspace(int64_t m, int64_t k, int64_t n, int64_t r, int dtype, int is_bwd);

int pf_lowrank_linear_gated_fwd(const void* x, int64_t ldx, const void* U, int64_t ldu, int64_t su,
                                const void* V, int64_t ldv, int64_t sv, const void* bias, int act,
                                void* y, int64_t ldy, void* T_stash, int64_t ldt, int64_t st,
                                int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                                void* workspace, size_t workspace_bytes, void* cuda_stream);

int pf_lowrank_linear_gated_bwd(const void* x, int64_t ldx, const void* U, int64_t ldu, int64_t su,
                                const void* V, int64_t ldv, int64_t sv, const void* bias, int act,
                                const void* dY, int64_t lddy, const void* T_stash, int64_t ldt, int64_t st,
                                void* dX, int64_t lddx, void* dU, int64_t lddu, int64_t sdu,
                                void* dV, int64_t lddv, int64_t sdv, void* dbias,
                                int64_t m, int64_t k, int64_t n, int64_t r, int dtype,
                                void* workspace, size_t workspace_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Log probabilities of given tokens at the end of a network, and what goes with them.  For each of `tokens` rows z of `vocab` logits (in `dtype`, pitch ld):
 *   lse = log sum exp(scale z)     log p = scale z - lse     entropy = - sum p log p     (fp32, each [tokens], NULL = not wanted)
 *   logprobs  log p of token ids[t] (int64); 0 for an id outside 0 .. vocab - 1 (padding)
 *   top       > 0: the `top` largest, in order, of equal ones (0 and -0 are equal) the one of the lowest id first:
 *             top_logprobs, top_ids (int64) [tokens, top], either NULL
 * Logits of -infinity have p = 0.  In a row that has no other, lse and all log probabilities are -infinity and the entropy is 0; a row that
 * holds a NaN or +infinity gives NaN (its top_ids count NaN as less than all numbers).
 * scale: 10^-6 .. 10^6, an inverse temperature.  ids NULL: no logprobs.
 * PF_ERR_UNSUPPORTED: a vocabulary of more than 819200 (PF_BF16) or 409600 (PF_F32), top > 128, 2^27 tokens.  One launch, no workspace.
 *
 * Backward, for the gradients dlogprobs and dentropy ([tokens] fp32, NULL = none; not both):
 *   dlogits = scale ( dlogprobs (1 at ids[t] - p) - dentropy p (log p + entropy) )      rounded once
 * where padding has no dlogprobs, and a row without a finite logit gets zeros.  dlogits may be logits (in place, with its pitch).  logprobs, entropy: as above,
 * from the same pass over the logits, for losses whose gradient is known beforehand.  The row's statistics are computed again: it is
 * read once and written once.
 * ------------------------------------------------------------------------------- */
int pf_logprobs_fwd(const void* logits, int64_t ld, const int64_t* ids, double scale, float* logprobs, float* entropy, float* lse,
                    int top, float* top_logprobs, int64_t* top_ids, int64_t tokens, int64_t vocab, int dtype, void* cuda_stream);

int pf_logprobs_bwd(const void* logits, int64_t ld, const int64_t* ids, double scale, const float* dlogprobs, const float* dentropy,
                    void* dlogits, int64_t lddl, float* logprobs, float* entropy,
                    int64_t tokens, int64_t vocab, int dtype, void* cuda_stream);

/* ---------------------------------------------------------------------------------
 * Divergence of a student's probabilities from a teacher's, of which the k largest logits were kept (a factorized network learns from the full-rank one
 * that it was made of).  teacher [tokens, k] fp32: logits (or log probabilities) of the tokens ids [tokens, k] (int64; outside 0 .. vocab - 1: no entry):
 *   q_j = exp(scale teacher_j - T),   T = log sum exp(scale teacher) over the row's entries, or teacher_lse [tokens] where that is given (over all of the
 *   teacher's logits, with the same scale)
 *   loss [tokens] (fp32) = sum over j of q_j (log q_j - log p of token ids_j)           p as for pf_logprobs_fwd, with the same scale
 * A token may stand in a row more than once (its entries add up).  Entries of -infinity have q = 0 and add nothing; a row without entries has the loss 0, a
 * token with q > 0 and a logit of -infinity makes it +infinity.
 * PF_ERR_UNSUPPORTED: k > 256, and sizes that pf_logprobs_fwd refuses.  One launch, no workspace.
 *
 * Backward, for dloss [tokens] fp32:  dlogits = scale dloss (p sum(q) - q at the entries' tokens), rounded once; in place and rows without a finite
 * logit as for pf_logprobs_bwd.  loss: as above from the same pass, NULL = not wanted.
 * ------------------------------------------------------------------------------- */
int pf_distill_fwd(const void* logits, int64_t ld, const int64_t* ids, const float* teacher, const float* teacher_lse, int k,
                   double scale, float* loss, int64_t tokens, int64_t vocab, int dtype, void* cuda_stream);

int pf_distill_bwd(const void* logits, int64_t ld, const int64_t* ids, const float* teacher, const float* teacher_lse, int k,
                   double scale, const float* dloss, void* dlogits, int64_t lddl, float* loss,
                   int64_t tokens, int64_t vocab, int dtype, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* PF_H_ */
