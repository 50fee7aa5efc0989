/*
 * libqvla -- the W4A4 quantized linear of Omega-QVLA (arxiv 2605.28803) on GB300 (sm_103a).
 *
 * The paper states the problem as Y ~= Delta_X' Delta_W' Q_X' Q_W' (Sec. 4.2, Eq. 7) after the
 * composite rotation X' = X P R_hat, W' = P^T R_hat^T W (Sec. 4.1, Eq. 3-5), with symmetric
 * int4 quantisation Delta = max|Z| / 7, Q = clamp(round(Z / Delta), -7, 7) (Sec. 4.2, Eq. 5-6),
 * weight scales per output channel, activation scales per token (backbone) or from a per-step
 * table indexed by the denoising step t (DiT head, Eq. 6 second display).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Matrices are row-major and dense.  Activations x are [M][K] (token-major), weights are
 *    stored [N][K] (output channel n in row n, y = x W^T), outputs y are [M][N].
 *  - Packed int4: byte j of a row holds code 2j in its low nibble and code 2j+1 in its high
 *    nibble, each a 4-bit two's-complement integer.  The quantiser only produces [-7, 7].
 *  - "device" pointers are CUDA global-memory addresses on the current device; "host"
 *    pointers are ordinary CPU memory.  The caller owns every buffer it passes in; the
 *    library owns what it allocates for a layer (packed weights, scales, bias, step table).
 *  - Calls taking a `stream` (a cudaStream_t passed as void*, NULL = legacy default stream)
 *    only enqueue work and return; they allocate nothing and never synchronise, so they can
 *    be captured in a CUDA graph.  All other calls are synchronous.
 *  - Every call returns a qvla_status.  On failure nothing was enqueued and
 *    qvla_last_error() returns a message for the calling thread.
 *  - Shapes: K % 128 == 0, the Hadamard block b is a power of two with 1 <= b <= 4096 and
 *    K % b == 0 (b == 1 disables the online rotation), N % 16 == 0, 0 <= M <= 1 << 20,
 *    K <= 16384 (so every integer accumulator is exact in float32).
 *  - Kernels wait on nothing without a time limit.  A wait that runs out records
 *    QVLA_ERR_TIMEOUT in a device-side word that qvla_check_device() reports.
 */
#ifndef QVLA_H
#define QVLA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  QVLA_OK = 0,
  QVLA_ERR_INVALID_ARG = 1,  /* a pointer, shape or dtype is not acceptable */
  QVLA_ERR_UNSUPPORTED = 2,  /* well-formed but outside what the kernels implement */
  QVLA_ERR_CUDA = 3,         /* a CUDA runtime call failed (message carries its text) */
  QVLA_ERR_OOM = 4,          /* device or host allocation failed */
  QVLA_ERR_STEP_RANGE = 5,   /* step t is outside [0, T) of the layer's table (or no table) */
  QVLA_ERR_TIMEOUT = 6       /* a device-side wait ran out of its time limit */
} qvla_status;

typedef enum { QVLA_F16 = 0, QVLA_BF16 = 1, QVLA_F32 = 2 } qvla_dtype;

/* Opaque device-resident layer: packed int4 weights, Delta_W, weight code sums, optional bias
 * and optional per-step table.  Created by qvla_pack_weights / qvla_layer_create. */
typedef struct qvla_layer qvla_layer;

/* Message describing the last failure on the calling thread ("" if none).  The pointer
 * stays valid until the next libqvla call on the same thread. */
const char* qvla_last_error(void);

/* Version of this interface; bumps on any incompatible change. */
int qvla_abi_version(void);

/* ------------------------------------------------------------------------------------------
 * Offline weight preparation (Sec. 4.1 Eq. 4-5; Sec. 4.2 Eq. 5-6 per output channel).  Host
 * only, touches no GPU.
 *
 * Folds the composite rotation into the weights, W'_n = W_n . P . BlockDiag(U_b) . BlockDiag(H_b)
 * (the [N][K] form of W' = P^T R_hat^T W), in float64; rounds W' once to float32; then per
 * output channel Delta_W[n] = max_k |W'[n,k]| / 7 (float32) and codes
 * clamp(round(W'/Delta_W), -7, 7), round half to even on the exact quotient.
 *
 *   W         host [N][K] of dtype wdt (F16, BF16 or F32).
 *   rot       host float64, NULL (U = I) or (K / rot_block) orthogonal blocks, each
 *             rot_block x rot_block row-major, block b acting on channels [b*rot_block, ...).
 *             A dense K x K factor is rot_block = K.  Orthogonality is the caller's promise.
 *   perm      host int32 [K] or NULL: column j of W.P is column perm[j] of W (a permutation).
 *   had_block Hadamard block b of the online rotation (the activations get the same block).
 *   wq        host out [N][K/2] packed codes.      wscale  host out [N] Delta_W (float32).
 *   wsum      host out [N] (may be NULL): sum over k of the weight codes of row n.
 * ------------------------------------------------------------------------------------------ */
qvla_status qvla_pack_weights_host(const void* W, qvla_dtype wdt, int N, int K,
                                   const double* rot, int rot_block, const int32_t* perm,
                                   int had_block, uint8_t* wq, float* wscale, int32_t* wsum);

/* The data-dependent factors of the composite rotation, chosen offline from the weights alone
 * (Sec. 4.1, Eq. 4 and the permutation P that follows it).  Host only.
 *   perm: input channels sorted by descending energy sum_n W[n,k]^2 (ties: lower channel
 *         first) and dealt across the K / block blocks in zigzag order -- forwards in even
 *         rounds, backwards in odd ones -- each block taking its channels in dealing order;
 *         column j of W.P is column perm[j] of W.
 *   rot:  for each block b of block channels of W.P, U_b = the block x block left singular
 *         vectors of the paper's row partition W_b = (W.P)[:, block b]^T, columns by
 *         descending singular value, each column's largest-magnitude entry positive; stored
 *         as qvla_pack_weights_host takes it (rot_block = block).
 * Pass both to qvla_pack_weights_host (with any Hadamard block that is a multiple of block) and
 * apply x . P . BlockDiag(U_b) to the activations upstream (reading: the library's online
 * rotation is the Hadamard factor).
 *   W     host [N][K] of dtype wdt.   block  divides K, 1 <= block <= 512.
 *   perm  host out int32 [K].          rot    host out float64 [K/block][block][block].
 * ------------------------------------------------------------------------------------------ */
qvla_status qvla_block_svd_rotation(const void* W, qvla_dtype wdt, int N, int K, int block, int32_t* perm,
                                    double* rot);

/* GPTQ-style weight codes (Sec. 5.1: the LLM side uses GPTQ with block size 128 and damping
 * ratio 0.01; the appendix on weight-quantisation solvers), written from the published GPTQ
 * algorithm.  Host only; a drop-in replacement of qvla_pack_weights_host's RTN codes with the
 * same fold, scales and packed layout.
 *   The weights are folded as in qvla_pack_weights_host and rounded to float32; Delta_W[n] is
 *   the RTN scale max |W'_n| / 7.  The n_cal calibration rows X (host [n_cal][K], dtype xdt,
 *   in the basis of W's input) are folded by the same P, U_b and Hadamard blocks, giving the
 *   Hessian H = 2/n_cal X'^T X'.  A column with H_kk = 0 is dead (its codes are 0); H gets
 *   damp * mean(diag H) on its diagonal.  With U the upper Cholesky factor of H^-1, the columns
 *   are quantised in order, q = clamp(round(w_i / Delta), +-7), and the error
 *   (w_i - Delta q) / U_ii is fed to every later column j times U_ij; updates beyond the current
 *   block of `block` columns are applied once per block (block = 128 in the paper).
 * Cost: O(K^3) for the factorisation and O(N K^2) for the codes (float64, all host cores);
 * memory 2 K^2 doubles.  Returns QVLA_ERR_INVALID_ARG if the damped Hessian is not positive
 * definite (e.g. damp = 0 with rank-deficient calibration data).
 *   block >= 1, damp >= 0, n_cal >= 1, K <= 16384; other arguments as qvla_pack_weights_host. */
qvla_status qvla_gptq_pack_host(const void* W, qvla_dtype wdt, int N, int K, const void* X, qvla_dtype xdt,
                                int n_cal, const double* rot, int rot_block, const int32_t* perm,
                                int had_block, int block, double damp, uint8_t* wq, float* wscale,
                                int32_t* wsum);

/* Upload already-packed weights as a layer (synchronous; allocates device memory the layer
 * owns).  wq host [N][K/2], wscale host [N], bias host [N] float32 or NULL.  xdt is the
 * activation dtype the layer accepts (F16, BF16 or F32); ydt the output dtype (F16 or BF16).
 * had_block as in qvla_pack_weights_host.  *out receives the layer. */
qvla_status qvla_layer_create(int N, int K, int had_block, qvla_dtype xdt, qvla_dtype ydt,
                              const uint8_t* wq, const float* wscale, const float* bias,
                              qvla_layer** out);

/* A gated-MLP layer: the gate and up projections of a backbone MLP (the Pi-0.5 / PaliGemma
 * backbone of Sec. 5.1), H output channels each, sharing one input.  They run as one GEMM whose
 * epilogue rounds gate and up to ydt like two stand-alone linears, then writes
 * h = ydt( gelu_tanh(gate) * up ), the input of the down projection.  The glue is the model's,
 * not the paper's method; it is fused here only to avoid storing gate and up.
 *   wq_gate, wq_up   host [H][K/2] packed codes (qvla_pack_weights_host of each projection)
 *   wscale_gate/_up  host [H];  bias_gate/_up host [H] float32 or NULL.
 * H % 128 == 0.  For this layer qvla_gemm_w4a4 and qvla_w4a4_linear write y as [M][H] (h),
 * and the optional acc output is [M][2H]: the H gate accumulators, then the H up ones. */
qvla_status qvla_layer_create_gated(int H, int K, int had_block, qvla_dtype xdt, qvla_dtype ydt,
                                    const uint8_t* wq_gate, const float* wscale_gate, const uint8_t* wq_up,
                                    const float* wscale_up, const float* bias_gate, const float* bias_up,
                                    qvla_layer** out);

/* qvla_pack_weights_host followed by qvla_layer_create (the spec entry point). */
qvla_status qvla_pack_weights(const void* W, qvla_dtype wdt, int N, int K,
                              const double* rot, int rot_block, const int32_t* perm,
                              int had_block, const float* bias, qvla_dtype xdt, qvla_dtype ydt,
                              qvla_layer** out);

/* Free a layer and everything it owns (synchronises the device first).  NULL is a no-op. */
qvla_status qvla_layer_destroy(qvla_layer* layer);

/* Per-step activation scale table of Eq. 6 (second display), read as one float32 per step
 * (per-tensor): scales host [T], each > 0 and finite, T >= 1.  Replaces any earlier table.
 * Synchronous. */
qvla_status qvla_set_step_scales(qvla_layer* layer, const float* scales, int T);

/* Per-step, per-group activation scales (Eq. 6 read per channel group; reading: one float32
 * per (step, group of max(128, had_block) channels) -- one k-block of the integer GEMM, or one
 * Hadamard block when that is larger).  scales host [T][G] with G = K / group (see
 * qvla_layer_scale_groups), each > 0 and finite.  Replaces any earlier table (per step or per
 * group).  With such a table, qvla_w4a4_linear at step t quantises channel k with
 * scales[t][k / group] and computes y = Delta_W[n] sum_g scales[t][g] acc_g[m,n] + bias[n],
 * acc_g the exact integer product over group g's channels: each group's accumulator is
 * corrected exactly and scaled before the float32 sum over the groups.  Not for gated layers
 * (QVLA_ERR_UNSUPPORTED); the other step-taking entry points refuse grouped tables with
 * QVLA_ERR_UNSUPPORTED (per-token calls, step == -1, are unaffected).  Synchronous. */
qvla_status qvla_set_step_group_scales(qvla_layer* layer, const float* scales, int T, int G);

/* Online data-dependent rotation for a layer whose activations cannot take x . P . BlockDiag(U_b)
 * upstream (Sec. 4.1, Eq. 4-5: layers that share one input but fold different P and U_b, such
 * as Q, K and V).  With it set, qvla_w4a4_linear, qvla_w4a4_linear_noalloc and
 * qvla_linear_quantize first form x' = x . P . BlockDiag(U_b) in the workspace -- float32
 * products summed in the order i = 0 .. rot_block - 1, one rounding to the activation dtype --
 * and run the Hadamard factor and the quantiser on x'; the workspace grows by M x K elements of
 * the activation dtype (qvla_linear_workspace_bytes accounts for it).  Pack the weights with the
 * same perm and rot (qvla_pack_weights_host).  qvla_rotate_quantize and qvla_w4a8_linear refuse
 * such a layer (QVLA_ERR_UNSUPPORTED).
 *   perm       host int32 [K] or NULL (identity): column j of x.P is column perm[j] of x.
 *   rot        host float64 [K/rot_block][rot_block][rot_block], row-major U_b (uploaded as
 *              float32), or NULL (U = I; perm alone).  Orthogonality is the caller's promise.
 *   rot_block  16, 32 or 64 (QVLA_ERR_UNSUPPORTED otherwise), dividing K.
 * perm == NULL and rot == NULL removes the online rotation.  Synchronous; the layer's device
 * must be current (QVLA_ERR_INVALID_ARG otherwise). */
qvla_status qvla_layer_set_online_rotation(qvla_layer* layer, const int32_t* perm, const double* rot, int rot_block);

/* The layer's online rotation alone: out = x . P . BlockDiag(U_b) as above (x, out device
 * [M][K] of the layer's activation dtype, distinct buffers), e.g. to calibrate step tables on the
 * values the quantiser sees.  QVLA_ERR_INVALID_ARG if the layer has no online rotation. */
qvla_status qvla_online_rotate(const qvla_layer* layer, const void* x, int M, void* out, void* stream);

/* The layer's scale groups: G groups of `group` channels (group = max(128, had_block)). */
qvla_status qvla_layer_scale_groups(const qvla_layer* layer, int* G, int* group);

/* Shape of a layer (N = output channels: H for a gated layer); any output pointer may be
 * NULL.  T is 0 when no table is set. */
qvla_status qvla_layer_info(const qvla_layer* layer, int* N, int* K, int* had_block, int* T);

/* ------------------------------------------------------------------------------------------
 * Online rotation + activation quantisation (Sec. 4.1 Eq. 5 online factor; Sec. 4.2 Eq. 5-6).
 *
 * For each row m of x (device [M][K], the layer's activation dtype, already in the P.U basis
 * applied upstream): y = x_m . BlockDiag(H_b/sqrt(b)) in float32, then
 *   step == -1 : per-token scale xscale[m] = max_k |y_k| / 7               (backbone)
 *   step >= 0  : xscale[m] = table[step] of the layer                        (DiT, Eq. 6)
 * and codes clamp(round(y / xscale[m]), -7, 7), round half to even on the exact quotient of
 * the float32 operands; xscale = 0 gives codes 0.  A NaN anywhere in row m makes its per-token scale NaN
 * (its codes then carry nothing), and so the linear's row m of y; a per-step scale clamps a NaN.
 *   xq      device out [M][K/2] packed codes.     xscale device out [M] float32.
 *   xsum    device out [M] int32 (may be NULL): sum over k of the codes of row m.  The GEMM
 *           needs it (its operand encoding is offset binary; the sum removes the offset).
 * Returns QVLA_ERR_STEP_RANGE for step outside [0, T) (or step >= 0 without a table).
 * ------------------------------------------------------------------------------------------ */
qvla_status qvla_rotate_quantize(const qvla_layer* layer, const void* x, int M, int step,
                                 uint8_t* xq, float* xscale, int32_t* xsum, void* stream);

/* The same operation without a layer, for any [M][K] input of dtype xdt and any block b
 * (b == 1: quantise x as given, no rotation).  step_scale is a DEVICE pointer to one float32
 * used as the per-step scale, or NULL for per-token scales. */
qvla_status qvla_rotate_quantize_rows(const void* x, qvla_dtype xdt, int M, int K, int had_block,
                                      const float* step_scale, uint8_t* xq, float* xscale,
                                      int32_t* xsum, void* stream);

/* Calibration helper for the per-step table (Eq. 6, sigma_hat = max abs): raises the device
 * float *absmax (which the caller initialises, e.g. to 0) to max |x . BlockDiag(H_b/sqrt(b))|
 * over all M x K entries.  The table entry is then absmax / 7. */
qvla_status qvla_rotated_absmax(const void* x, qvla_dtype xdt, int M, int K, int had_block,
                                float* absmax, void* stream);

/* The same calibration per scale group: absmax device [K / group] floats (group =
 * max(128, had_block), K a multiple of it), entry g raised to the max over the M rows and the
 * group's channels.  The per-group table entry is then absmax[g] / 7. */
qvla_status qvla_rotated_absmax_groups(const void* x, qvla_dtype xdt, int M, int K, int had_block,
                                       float* absmax, void* stream);

/* ------------------------------------------------------------------------------------------
 * Integer GEMM + dequantisation epilogue (Sec. 4.2 Eq. 7, scales "folded into
 * dequantization", Sec. 5.1):
 *   acc[m,n] = sum_k xq[m,k] * wq[n,k]                       (exact integer)
 *   y[m,n]   = ydt( fma( (float)acc[m,n], xscale[m] * Delta_W[n], bias[n] ) )
 * with xscale[m] * Delta_W[n] one float32 product, the fma in float32 and one
 * round-to-nearest-even conversion to the layer's output dtype.
 *   xq device [M][K/2], xscale device [M], xsum device [M] (from qvla_rotate_quantize),
 *   y device out [M][N] of the layer's output dtype,
 *   acc device out [M][N] int32, or NULL (debug/test hook: the exact integer accumulator);
 *       16-byte aligned like xq and y.
 * ------------------------------------------------------------------------------------------ */
qvla_status qvla_gemm_w4a4(const qvla_layer* layer, const uint8_t* xq, const float* xscale,
                           const int32_t* xsum, int M, void* y, int32_t* acc, void* stream);

/* Bytes of device workspace qvla_w4a4_linear takes for M rows (a multiple of 256): the codes
 * travel between its two kernels as one tensor-core operand byte each (M x K bytes), plus the
 * scales, the code sums and the per-group code sums (M x G x 4 bytes), and, for a layer with an
 * online rotation, x . P . BlockDiag(U_b) (M x K elements of the activation dtype).  Where the
 * GEMM's tiles could leave SMs idle (M > 128, not gated, fewer 128 x 256 tiles than SMs) it adds
 * room for splitting each tile's K into up to 4 work units: 4 FP32 partials per output (M and N
 * rounded up to 256) and 4 bytes of counter per 128 x 128 tile.  The linear also runs in a
 * workspace of the first parts only; its GEMM then does not split K. */
size_t qvla_linear_workspace_bytes(const qvla_layer* layer, int M);

/* The whole online linear (Sec. 4): rotate + quantise x (as qvla_rotate_quantize, step as
 * there), then the integer GEMM and epilogue (as qvla_gemm_w4a4).  x device [M][K], y device
 * out [M][N].  workspace: caller-owned device memory of at least
 * qvla_linear_workspace_bytes(layer, M) bytes, 256-byte aligned, used only during the call's
 * kernels on `stream` (calls that overlap on the GPU must not share it).
 * One token (M = 1, the decode step) runs as a single kernel where the layer allows it (f16 or
 * bf16 input of the output's dtype, Hadamard block <= 2048, no per-group step table, a split of
 * K whose CTAs each see at most two 2048-channel rotation passes): a GEMV whose CTAs rotate and
 * quantise their share of x themselves, with the same results bit for bit; the workspace is
 * then not touched unless the layer has an online rotation. */
qvla_status qvla_w4a4_linear(const qvla_layer* layer, const void* x, int M, int step, void* y,
                             void* workspace, size_t workspace_bytes, void* stream);

/* The one-launch linear for a small batch with a per-step scale: the rotation, the quantiser, the
 * integer GEMM and the epilogue of qvla_w4a4_linear (same arithmetic, same results) in a single
 * kernel -- the DiT head's case (Sec. 4.2, Eq. 6: the scale is the step's table entry, so no
 * reduction along a row precedes the quantiser).  The CTAs that split the reduction over K
 * rotate and quantise the token rows among themselves and exchange the codes in shared memory;
 * nothing goes through a workspace.  Every CTA of a cluster rotates whole token rows, so each
 * weight tile's cluster repeats the rotation of all M rows: on GB300 this takes longer than the
 * two launches of qvla_w4a4_linear at every DiT shape measured except K = 512 at M = 1, and
 * qvla_w4a4_linear does not use it.  x device [M][K] (f16 or bf16), y device out [M][N], step in
 * [0, T).
 * QVLA_ERR_UNSUPPORTED (nothing enqueued) where it does not apply: step == -1, M > 128, K outside
 * [512, 4096] or not a multiple of the task width (512 channels up to K = 512, 1024 up to 1024,
 * 2048 beyond), activation and output dtypes that differ or are f32, gated layers, per-group
 * tables, an online P.U, or no split of K whose tiles fit the kernel's shared memory. */
qvla_status qvla_w4a4_linear_fused(const qvla_layer* layer, const void* x, int M, int step, void* y, void* stream);

/* The two halves of qvla_w4a4_linear, for callers that schedule them separately (for example to
 * time them, or to overlap one layer's GEMM with the next layer's rotation on another stream).
 * qvla_linear_quantize rotates and quantises x into `workspace` (as qvla_rotate_quantize, step
 * as there); qvla_linear_gemm then runs the integer GEMM and epilogue on it (as qvla_gemm_w4a4).
 * The workspace contents in between are internal to the library: the codes as tensor-core
 * operand bytes, the scales and the code sums, which the GEMM only reads, and the counters of
 * the GEMM's split of K, which qvla_linear_quantize zeroes and the GEMM leaves zero (it uses the
 * split's room as scratch).  So qvla_linear_gemm must follow a qvla_linear_quantize of the same
 * layer, M and workspace; it may run again on the same codes.  Same workspace rules as
 * qvla_w4a4_linear. */
qvla_status qvla_linear_quantize(const qvla_layer* layer, const void* x, int M, int step, void* workspace,
                                 size_t workspace_bytes, void* stream);
qvla_status qvla_linear_gemm(const qvla_layer* layer, void* workspace, size_t workspace_bytes, int M, void* y,
                             void* stream);

/* Allocation-free variant of qvla_w4a4_linear.  The paper has no counterpart: this entry
 * point exists for callers that must not allocate device memory once they are running --
 * for example a robot controller's real-time loop, which reserves all of its memory at start-up
 * because an allocation inside the loop can stall for milliseconds or fail mid-episode, or a
 * plug-in whose host runtime hands out device memory only from its own pool.  Such a caller
 * cannot provide qvla_w4a4_linear's workspace on demand, so this call uses a fixed scratch area
 * that the library itself holds instead.
 *
 * The scratch is one file-scope device array of QVLA_NOALLOC_SCRATCH_BYTES (8 MiB).  Every GPU
 * that loads the library holds it until the process exits.  The call allocates nothing: it
 * makes no cudaMalloc/cudaFree and calls no allocating library routine.  Its first call on each
 * device looks up the array's device address with that device current; make that first call
 * before any stream capture.  The scratch must hold qvla_linear_workspace_bytes(layer, M)
 * bytes, each part rounded up to a multiple of 256: the codes as operand bytes (M x K), the
 * scales and the code sums (M x 4 each), the per-group code sums (M x G x 4, G = K / max(128,
 * had_block)) and, for a layer with an online rotation, x . P . BlockDiag(U_b) (M x K elements
 * of the activation dtype).  Larger requests fail with QVLA_ERR_UNSUPPORTED and enqueue
 * nothing.  The layer must live on the current device (QVLA_ERR_INVALID_ARG otherwise).  Every call shares the one array and leaves the
 * last call's contents in it; each call overwrites all it reads, so nothing needs clearing
 * in between.  Two calls whose kernels overlap on the GPU (different streams or threads, on
 * the same device) race on the array: issue them on one stream.
 * Arguments and results are those of qvla_w4a4_linear without the workspace. */
#define QVLA_NOALLOC_SCRATCH_BYTES ((size_t)8 << 20)
qvla_status qvla_w4a4_linear_noalloc(const qvla_layer* layer, const void* x, int M, int step, void* y,
                                     void* stream);

/* ------------------------------------------------------------------------------------------
 * W4A8 variant (the appendix on the real-quantization kernel, "Real-Quantization Kernel
 * Implementation", Table 5): the same int4 weights of the layer against 8-bit activation codes,
 * with the same scales and epilogue.  Per token (step == -1) the scale is max_k |y_k| / 127;
 * per step it is the table entry as given (a table calibrated for 8-bit codes holds
 * absmax / 127); codes are clamp(round(y / xscale[m]), -127, 127), round half to even on the
 * exact quotient of the float32 operands.  With had_block == 1 no rotation runs at all, the
 * appendix's configuration (rotations folded into the weights offline).
 *
 * The accumulator stays exact for K <= 4096 (255 x 15 x K < 2^24 units of the tensor cores'
 * float32 accumulator); layers with a longer K return QVLA_ERR_UNSUPPORTED.
 * ------------------------------------------------------------------------------------------ */

/* Rotate + quantise to 8-bit codes: as qvla_rotate_quantize_rows with q_max = 127.
 *   xq device out [M][K] int8 codes, natural k order, 16-byte aligned.
 *   xscale device out [M] float32; xsum device out [M] int32 or NULL (sum of row m's codes). */
qvla_status qvla_rotate_quantize_rows_a8(const void* x, qvla_dtype xdt, int M, int K, int had_block,
                                         const float* step_scale, int8_t* xq, float* xscale,
                                         int32_t* xsum, void* stream);

/* Bytes of device workspace qvla_w4a8_linear and qvla_gemm_w4a8 need for M rows (a multiple of
 * 256): the codes as two tensor-core operand planes (M x 2K bytes), the scales and the sums. */
size_t qvla_w4a8_workspace_bytes(const qvla_layer* layer, int M);

/* The whole W4A8 linear: rotate + quantise x to 8-bit codes (step as in qvla_rotate_quantize),
 * then the integer GEMM and the epilogue of qvla_gemm_w4a4 on them.  x device [M][K], y device
 * out [M][N] (H for a gated layer); workspace as for qvla_w4a4_linear but of
 * qvla_w4a8_workspace_bytes(layer, M) bytes. */
qvla_status qvla_w4a8_linear(const qvla_layer* layer, const void* x, int M, int step, void* y,
                             void* workspace, size_t workspace_bytes, void* stream);

/* Integer GEMM + epilogue on 8-bit codes quantised elsewhere (e.g. by
 * qvla_rotate_quantize_rows_a8):  acc[m,n] = sum_k xq[m,k] * wq[n,k] (exact),
 * y[m,n] = ydt(fma((float)acc[m,n], xscale[m] * Delta_W[n], bias[n])).
 *   xq device [M][K] int8 (16-byte aligned), xscale device [M];
 *   y device out, acc device out [M][N] int32 or NULL (test hook), as in qvla_gemm_w4a4;
 *   workspace of qvla_w4a8_workspace_bytes(layer, M) bytes, 256-byte aligned (the operand
 *   planes and the code sums are built there first). */
qvla_status qvla_gemm_w4a8(const qvla_layer* layer, const int8_t* xq, const float* xscale, int M, void* y,
                           int32_t* acc, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Attention between the quantised linears, and a key/value cache of 4-bit codes.
 *
 * The paper quantises the linears of the language backbone and of the DiT action head (Sec. 5.1);
 * what runs between the fused Q/K/V linear and the output linear is the model's softmax attention
 *     o_i = sum_j p_ij v_j,   p_ij = exp(scale q_i.k_j) / sum_j' exp(scale q_i.k_j'),
 * j over the keys that query i sees.  Conventions of the calls below:
 *  - A token's heads are contiguous: element (t, h, c) of q is q[t * q_stride + h * head_dim + c],
 *    so q, k and v may be slices of the fused linear's output (q_stride its row length).  Strides
 *    are in elements, multiples of 8 and at least heads * head_dim (kv_heads * head_dim); pointers
 *    are 16-byte aligned.  Outputs are dense: o[t][heads][head_dim].
 *  - dt is QVLA_F16 or QVLA_BF16, for queries, keys, values and outputs alike.  head_dim is 64, 128
 *    or 256; kv_heads divides heads, and query head h reads key/value head h / (heads / kv_heads).
 *  - Sequences are packed: sequence b's queries are rows [cu_q[b], cu_q[b+1]) (device int32
 *    [batch + 1], not decreasing).  Lengths may be zero and may change between replays of a CUDA
 *    graph within total_q / total_k.
 *  - causal != 0: with n queries and m keys, query i of its sequence sees keys 0 .. m - n + i (the last
 *    query stands at the last key).  A query that sees no key (m == 0, or m - n + i < 0) gets zeros.
 *    A key or value that a query does not see has no effect on it, whatever its bits (NaN, Inf).
 *  - scale is positive and finite (1 / sqrt(head_dim) as a rule).  Scores, the softmax's maximum
 *    and sum, and the sum over the values are held in float32.
 *  - Indices in device memory (cu_q, cu_k, page tables, lengths) that leave the buffers they index are
 *    caught on the device: the tokens concerned are skipped, and qvla_check_device() reports
 *    QVLA_ERR_INVALID_ARG.  Offsets below 0 or beyond total_q / total_k are cut off, a sequence whose
 *    offsets decrease has no tokens, and either is reported too.
 * ------------------------------------------------------------------------------------------ */

/* Attention over packed prompts.
 *   q [total_q], k and v [total_k] tokens as above; cu_k device int32 [batch + 1], may be cu_q.
 *   o device out [total_q][heads][head_dim]; rows outside every sequence are not written.
 * batch in [0, 65535], total_q and total_k in [0, 2^24], heads <= 1024.
 * The probabilities are rounded to dt for the product with the values. */
qvla_status qvla_attention_prompt(const void* q, const void* k, const void* v, qvla_dtype dt, int heads, int kv_heads,
                                  int head_dim, int64_t q_stride, int64_t k_stride, int64_t v_stride, int batch,
                                  const int32_t* cu_q, int total_q, const int32_t* cu_k, int total_k, float scale,
                                  int causal, void* o, void* stream);

/* A paged key/value cache of 4-bit codes in one device buffer of the caller (the pool).
 *   pool      device, 16-byte aligned, qvla_kv4_pool_bytes(...) bytes: num_pages x kv_heads blocks of
 *             page_size * (head_dim + 8) bytes, each holding, for one head's tokens of the page, the key
 *             codes [page_size][head_dim / 2], the value codes (the same), the key scales float32
 *             [page_size] and the value scales.  Byte j of a token's codes holds channel 2j in its
 *             low nibble and 2j + 1 in its high nibble, two's complement in [-7, 7].
 *   page_size 16, 32, 64, 128 or 256 tokens.
 *   rotate    nonzero: every head is multiplied by H / sqrt(head_dim) (H the Sylvester Hadamard matrix)
 *             ahead of the quantiser, which spreads a head's large channels (Sec. 4.1 Eq. 3, applied
 *             to the cached heads).  Queries are rotated alike, and outputs rotated back.
 * A token's head has one scale, Delta = max |y| / 7 (rounded to float32), and codes clamp(round(y / Delta),
 * -7, 7), round half to even on the exact quotient of the float32 numbers (Sec. 4.2 Eq. 5-6 per token and
 * head); Delta = 0 gives codes 0.
 * A head with a NaN or an infinity reads back as NaN.
 * A sequence's tokens lie at positions 0, 1, 2, ...; position p of sequence b is slot p % page_size of
 * page page_table[b * max_pages + p / page_size] (device int32 [batch][max_pages]). */
typedef struct {
  void* pool;
  int num_pages;
  int page_size;
  int kv_heads;
  int head_dim;
  int rotate;
} qvla_kv4_cache;

/* Bytes of a pool; 0 for a geometry that the calls below refuse. */
size_t qvla_kv4_pool_bytes(int num_pages, int page_size, int kv_heads, int head_dim);

/* Quantise new tokens' keys and values into the cache: token t of sequence b, at row cu_new[b] + t of k
 * and v, goes to position start[b] + t (start device int32 [batch]: the tokens cached before; NULL: 0).
 * Two rows of one call must not name the same slot. */
qvla_status qvla_kv4_append(const qvla_kv4_cache* cache, const void* k, const void* v, qvla_dtype dt, int64_t k_stride,
                            int64_t v_stride, int batch, const int32_t* cu_new, int total_new,
                            const int32_t* page_table, int max_pages, const int32_t* start, void* stream);

/* Read cached tokens back, in the model's basis (rotated back) and rounded to dt: position start[b] + t
 * (start NULL: 0) of sequence b to row cu[b] + t of k and v (device out [total][kv_heads][head_dim]),
 * for example as the first part of a prompt's keys and values for qvla_attention_prompt.  A position
 * without a page gives zeros. */
qvla_status qvla_kv4_gather(const qvla_kv4_cache* cache, int batch, const int32_t* cu, int total,
                            const int32_t* page_table, int max_pages, const int32_t* start, void* k, void* v,
                            qvla_dtype dt, void* stream);

/* Bytes of workspace that let qvla_attention_kv4 split the keys of each sequence as far as is useful on the
 * current device (a multiple of 256; 0 when no split would be made). */
size_t qvla_attention_kv4_workspace_bytes(int heads, int kv_heads, int head_dim, int batch, int total_q, int max_q,
                                          int max_len);

/* Attention of a few query tokens of every sequence over its cached keys and values: one token while
 * decoding, a chunk of action tokens, a few speculated tokens.  The codes are multiplied as they are and
 * the scales applied to scores and probabilities; nothing is written back to memory as values.
 *   q          [total_q] tokens, total_q * heads < 2^31 - 16;  max_q >= the queries of any sequence, at most 2^24
 *   kv_len     device int32 [batch]: cached tokens of each sequence (with causal != 0 the queries' own
 *              tokens, appended before, are the last of them);  max_len >= every kv_len, at most 2^30.  max_q and
 *              max_len shape the launch: a sequence that exceeds them is skipped, and reported by
 *              qvla_check_device().
 *   o          device out [total_q][heads][head_dim]
 *   workspace  device, 256-byte aligned, or NULL with 0 bytes: room for the partial results of a split
 *              over the keys (qvla_attention_kv4_workspace_bytes; a smaller one allows a smaller split).
 *              Used only during the call's kernels on `stream`.
 * Each probability times its value scale is rounded to float16 against a power of two that follows the
 * row's largest (11 bits whatever the scales' size); queries are rounded to float16 likewise. */
qvla_status qvla_attention_kv4(const qvla_kv4_cache* cache, const void* q, qvla_dtype dt, int heads, int64_t q_stride,
                               int batch, const int32_t* cu_q, int total_q, int max_q, const int32_t* page_table,
                               int max_pages, const int32_t* kv_len, int max_len, float scale, int causal, void* o,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Microscaled 4-bit floating point: the linear with codes that sm_103a's tensor cores take as they are.
 *
 * A code is E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 (0 to 7) and their negatives (bit 3); byte j of a row holds code 2j in its low
 * nibble and 2j + 1 in its high one.  Consecutive channels share a block scale:
 *   QVLA_MXFP4  32 channels, E8M0 (byte b: 2^(b - 127), 255 NaN).
 *               e = floor(log2 max |z|) - 2, at least -127; codes E2M1(z / 2^e), values above 6 becoming 6.
 *   QVLA_NVFP4  16 channels, E4M3, and a float32 scale Delta of the row.
 *               Delta = max_row |z| / 2688 (rounded to float32), or the step's scale; s = E4M3(max_block |z| / (6 Delta)), at most
 *               448; codes E2M1(z / D), D = s Delta rounded to float32; an entry stands for code * s * Delta.
 * Roundings are to nearest, ties to the even code, decided on the exact quotient of the float32 numbers.  z is the row, or with
 * had_block > 1 the row times BlockDiag(H_b / sqrt(b)) (Sec. 4.1 Eq. 3): float32 butterflies of distance b/2, b/4, ..., 1,
 * then one float32 product.  A block of zeros has codes 0 (of either sign) and scale 0.  A row with a NaN or an infinity has
 * no finite meaning: an MX block that holds one has scale 255; in NV it makes Delta NaN, and with a step's scale a NaN
 * makes its block's scale NaN and an infinity is clamped.
 *   Block scales lie in tiles of 128 rows x 4 blocks, 512 bytes each, tile (m / 128, b / 4) of a row-major grid of
 * ceil(rows / 128) x (blocks / 4): the scale of row m and block b is byte (m % 32) * 16 + (m / 32 % 4) * 4 + b % 4 of its tile.
 * Bytes of rows past the last one are neither written nor used.  Shapes as above: K % 128 == 0, K <= 16384, N % 16 == 0, b up to 4096.
 * ------------------------------------------------------------------------------------------ */
typedef enum { QVLA_MXFP4 = 0, QVLA_NVFP4 = 1 } qvla_fp4_format;

/* Bytes of the block scales of `rows` rows; 0 for a format or shape that the calls below refuse. */
size_t qvla_fp4_scale_bytes(qvla_fp4_format fmt, int rows, int K);

/* Rotate and quantise rows.  x device [M] rows of K, x_stride elements apart (a multiple of 8, at least K; x 16-byte aligned).
 *   step_scale  device, one positive float32 in the place of every row's Delta, or NULL (NULL for MX)
 *   xq          device out [M][K/2], 16-byte aligned;  xs  device out, 16-byte aligned, qvla_fp4_scale_bytes(fmt, M, K) bytes
 *   xscale      device out [M] float32: Delta.  Not touched for MX, and may be NULL then. */
qvla_status qvla_fp4_quantize_rows(const void* x, qvla_dtype xdt, int64_t x_stride, int M, int K, int had_block,
                                   qvla_fp4_format fmt, const float* step_scale, uint8_t* xq, uint8_t* xs, float* xscale,
                                   void* stream);

/* What the codes stand for, in the rotated basis: code * block scale * Delta in float32, rounded to odt (F16, BF16 or F32).
 *   out device [M][K], 16-byte aligned; xscale is not read for MX. */
qvla_status qvla_fp4_dequantize_rows(const uint8_t* xq, const uint8_t* xs, const float* xscale, qvla_fp4_format fmt, int M,
                                     int K, void* out, qvla_dtype odt, void* stream);

/* Fold and quantise weights on the host: the fold is qvla_pack_weights_host's (P, U_b and the Hadamard block in float64, one
 * rounding to float32), the codes those of a row above.
 *   wq host out [N][K/2];  ws host out, qvla_fp4_scale_bytes(fmt, N, K) bytes (bytes of no row become 0);
 *   wscale host out [N] float32: Delta of each output channel.  Not touched for MX, and may be NULL then. */
qvla_status qvla_fp4_pack_weights_host(const void* W, qvla_dtype wdt, int N, int K, const double* rot, int rot_block,
                                       const int32_t* perm, int had_block, qvla_fp4_format fmt, uint8_t* wq, uint8_t* ws,
                                       float* wscale);

/* A device-resident layer of such weights.  Its device must be current in the calls that take it (QVLA_ERR_INVALID_ARG). */
typedef struct qvla_fp4_layer qvla_fp4_layer;

/* Upload packed weights (synchronous; the layer owns what it allocates).  Arrays as qvla_fp4_pack_weights_host writes them;
 * wscale NULL for MX; bias host [N] float32 or NULL.  xdt (F16, BF16 or F32) is what qvla_fp4_linear takes, ydt (F16 or BF16)
 * the output.  A NaN or negative block scale, or a wscale that is not finite and non-negative, is refused. */
qvla_status qvla_fp4_layer_create(int N, int K, int had_block, qvla_fp4_format fmt, qvla_dtype xdt, qvla_dtype ydt,
                                  const uint8_t* wq, const uint8_t* ws, const float* wscale, const float* bias,
                                  qvla_fp4_layer** out);

/* The gate and up projections of a gated MLP as one layer, H output channels (H % 128 == 0): the arrays hold 2H rows, H gate
 * rows and then H up rows.  Its output is ydt(gelu_tanh(gate) * up) [M][H], gate and up in float32. */
qvla_status qvla_fp4_layer_create_gated(int H, int K, int had_block, qvla_fp4_format fmt, qvla_dtype xdt, qvla_dtype ydt,
                                        const uint8_t* wq, const uint8_t* ws, const float* wscale, const float* bias,
                                        qvla_fp4_layer** out);

/* Free a layer (synchronises the device first).  NULL is a no-op. */
qvla_status qvla_fp4_layer_destroy(qvla_fp4_layer* layer);

/* The product of quantised rows and a layer: y[m,n] = ydt(fma(acc, xscale[m] * wscale[n], bias[n])), acc the float32 sum over
 * k of (code * block scale) of both; with MX xscale and wscale are 1.
 *   xq, xs, xscale  as qvla_fp4_quantize_rows writes them (16-byte aligned; xscale is not read for MX)
 *   y               device out [M][N] (gated: [M][H]) of ydt, 16-byte aligned
 * The sums' order depends on the call's sizes; the same call gives the same bits. */
qvla_status qvla_gemm_fp4(const qvla_fp4_layer* layer, const uint8_t* xq, const uint8_t* xs, const float* xscale, int M,
                          void* y, void* stream);

/* Bytes of device workspace of qvla_fp4_linear for M rows (a multiple of 256). */
size_t qvla_fp4_linear_workspace_bytes(const qvla_fp4_layer* layer, int M);

/* The whole linear: the layer's rotation and quantiser on x (device [M][K] of xdt, dense), then the product.  step_scale as
 * in qvla_fp4_quantize_rows; workspace as in qvla_w4a4_linear.  y may overlap x.  Up to 4 tokens are one launch where x has y's type
 * and does not overlap it, and the workspace may then be left as it was. */
qvla_status qvla_fp4_linear(const qvla_fp4_layer* layer, const void* x, int M, const float* step_scale, void* y,
                            void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * What runs between two blocks (attention, MLP) of a layer: the residual takes a block's output, gated and normalised where
 * the model does so, and the next block's input is the residual's norm, modulated where the model conditions it.
 *   u  = y, or with post_norm != 0  norm(y) * (post_weight + weight_offset)
 *   r' = residual_scale * r + gate * u                         rounded to the residual's type, stored
 *   h  = (norm(r') * (pre_weight + weight_offset) + pre_bias) * (1 + scale) + shift     rounded to dt
 * with norm(x) = x / sqrt(mean(x^2) + eps)                 (QVLA_NORM_RMS)
 *        norm(x) = (x - mean x) / sqrt(mean((x - mean x)^2) + eps)  (QVLA_NORM_LAYER)
 * in float32 over a row's K channels.  A norm reads r' as it is stored.  A factor or term whose pointer is NULL is left out.
 * Squares that leave float32's range make a row's norm 0 or NaN.
 * ------------------------------------------------------------------------------------------ */
typedef enum { QVLA_NORM_RMS = 0, QVLA_NORM_LAYER = 1 } qvla_norm_kind;

typedef struct {
  qvla_norm_kind kind;      /* of both norms */
  float eps;                /* positive */
  float weight_offset;      /* added to both weights: 1 where a model stores them less one */
  float residual_scale;
  int post_norm;
  const void* post_weight;  /* device [K] of dt, as pre_weight and pre_bias, or NULL */
  const void* pre_weight;
  const void* pre_bias;
  const void* gate;         /* device, mod_rows rows of K of dt, mod_stride elements apart (a multiple of 8), or NULL */
  const void* scale;
  const void* shift;
  int64_t mod_stride;
  int mod_rows;
  int mod_tokens;             /* token m takes row m / mod_tokens, */
  const int32_t* mod_index;   /* or, where this is not NULL, row mod_index[m] (device int32 [M]): a token whose row is not
                                 in [0, mod_rows) is skipped, nothing of it is written, and qvla_check_device() reports
                                 QVLA_ERR_INVALID_ARG */
} qvla_block_norm_params;

/* One junction with its output in 16 bits.
 *   r  device [M] rows of K of rdt (dt, or F32), r_stride elements apart (a multiple of 8)
 *   y  device, the block's output, rows of dt y_stride elements apart, or NULL: no block has run yet
 *   r_out  device, rows r_stride apart; may be r.  NULL where y is NULL and residual_scale is 1: r is left as it is
 *   h  device out [M][K] of dt (F16 or BF16), dense, or NULL: the residual alone
 * Pointers are 16-byte aligned; K % 8 == 0, K <= 16384, M in [0, 2^20].  h and r_out overlap no input, but r_out may be r
 * itself, and h may be y itself where y_stride is K or M is 1 (QVLA_ERR_INVALID_ARG else). */
qvla_status qvla_block_norm(const qvla_block_norm_params* norm, qvla_dtype dt, const void* r, qvla_dtype rdt, int64_t r_stride,
                            const void* y, int64_t y_stride, int M, int K, void* r_out, void* h, void* stream);

/* The same with h rotated and quantised as by qvla_fp4_quantize_rows (which it equals, on h rounded to dt): hq, hs and hscale
 * are that call's xq, xs and xscale.  h may be NULL.  K % 128 == 0. */
qvla_status qvla_block_norm_fp4(const qvla_block_norm_params* norm, qvla_dtype dt, const void* r, qvla_dtype rdt,
                                int64_t r_stride, const void* y, int64_t y_stride, int M, int K, void* r_out, void* h,
                                int had_block, qvla_fp4_format fmt, const float* step_scale, uint8_t* hq, uint8_t* hs,
                                float* hscale, void* stream);

/* Synchronise `stream`, then report (and clear) the device-side error words: QVLA_OK,
 * QVLA_ERR_TIMEOUT if a kernel gave up waiting since the last check, or QVLA_ERR_INVALID_ARG if an
 * attention, cache or norm kernel met an index in device memory that it had to skip. */
qvla_status qvla_check_device(void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QVLA_H */
