/*
 * libqgalore - the per-weight-matrix Q-GaLore optimizer step for AMD MI355X (gfx950).
 *
 * C ABI.  Conventions that hold for every entry point unless stated otherwise:
 *
 *  - Every data pointer is a DEVICE pointer owned by the caller.  The library
 *    never allocates, frees or retains device memory; scratch space is passed
 *    in as `workspace` (size from the matching *_workspace_bytes query).
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *    Calls enqueue work and return WITHOUT synchronising.
 *  - All matrices are dense row-major with leading dimension = row length
 *    (the *_ld entry points and the grouped descriptors take a row pitch).
 *    Base pointers must be 16-byte aligned (QG_ERR_ALIGN otherwise).
 *  - Notation (the paper's): W is the m x n weight, G the m x n gradient,
 *    P the m x r projection matrix, R = P^T G (r x n), M and V the Adam moments
 *    (r x n), N the Adam direction (r x n), U = alpha P N (m x n), t the 1-based
 *    step count.
 *  - `group` is the quantization block size; only 256 (the paper's value,
 *    Sec. 3.1) is accepted, anything else returns QG_ERR_GROUP.
 *  - INT8 weight format: codes int8 [m][n]; one fp32 scale per block of 256
 *    consecutive elements OF A ROW, scales [m][ceil(n/256)] (a row's last block
 *    is short when n % 256 != 0).  Symmetric: zero point 0, scale = absmax/127.
 *  - INT4 projection format: block = 256 consecutive elements of the FLATTENED
 *    row-major m x r array, scales [ceil(m*r/256)], scale = absmax/7.  Two
 *    codes per byte, flat element 2b in the low nibble of byte b, stored
 *    nibble = code + 8.
 *  - bf16 tensors are passed as uint16_t bit patterns.
 *  - Sizes are positive: an empty tensor (m, n, r or an element count of 0) is
 *    an argument error (QG_ERR_SHAPE), not a no-op; m * n must stay below 2^32
 *    (the stochastic-rounding stream and the kernels index elements with 32
 *    bits), r is a multiple of 8 and at most m.
 *  - Return value: QG_OK or a QG_ERR_* code.  Arguments are validated before
 *    any HIP call, so argument errors are reported even with no GPU present.
 *    After QG_ERR_HIP, qg_last_hip_error() returns the hipError_t value.
 */
#ifndef QGALORE_H
#define QGALORE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    QG_OK = 0,
    QG_ERR_NULL = 1,       /* a required pointer is NULL */
    QG_ERR_SHAPE = 2,      /* m, n, r, count, step out of range (see each call) */
    QG_ERR_GROUP = 3,      /* group != 256 */
    QG_ERR_ALIGN = 4,      /* a base pointer is not 16-byte aligned */
    QG_ERR_WORKSPACE = 5,  /* workspace missing or too small */
    QG_ERR_HIP = 6         /* a HIP call or kernel launch failed */
};

/* Adam and GaLore hyper-parameters (Sec. 4.1: Adam as the inner optimizer,
 * scale factor alpha = 0.25). */
typedef struct {
    float beta1, beta2, eps, lr, alpha;
} qg_hparams;

/* Per-layer state of the adaptive lazy subspace update (Sec. 3.2). */
typedef struct {
    int interval;      /* current refresh interval t (steps) */
    int streak;        /* consecutive checks with cos >= threshold */
    int k;             /* checks in a row required before the interval doubles */
    int next_refresh;  /* step at which the next refresh is due */
    float threshold;   /* 0.4 in the paper */
    float last_cos;
} qg_policy;

/* One matrix of a grouped step (qg_step_many).  All pointers are device
 * pointers with the layouts of the single-matrix calls, except for the optional row pitch `ld`. */
typedef struct {
    int64_t m, n, r;
    const uint8_t*  Pq;   /* INT4 P, packed            */
    const float*    Ps;   /* INT4 P block scales        */
    const uint16_t* G;    /* bf16 gradient m x n        */
    int8_t*         Wq;   /* INT8 weight codes, in/out  */
    float*          Ws;   /* INT8 weight scales, in/out */
    float*          M;    /* first moment r x n, in/out */
    float*          V;    /* second moment r x n, in/out*/
    float*          R;    /* projected gradient r x n, out; may be NULL (not written then) */
    uint16_t*       N;    /* bf16 Adam direction r x n, out */
    int64_t         ld;   /* row pitch, in elements, of EVERY n-wide array above (G, Wq: m rows; M, V, R, N: r rows).
                             0 or n: dense rows.  Otherwise >= n and a multiple of 16: rows then start 16-byte aligned
                             whatever n is, which takes a matrix with n % 8 != 0 (n = 5461 in the LLaMA-1B shapes) off
                             the slow under-aligned path.  Every array holds rows * ld elements.  Padding columns are never read for a
                             result; they are not written either, except that the unfused
                             qg_lowrank_adam_many runs over the padding of M, V, N as well. */
    float*          Wz;   /* zero points of W, [m][ceil(n/256)], in/out, or NULL: the symmetric format.  Either every
                             matrix of a plan has them or none (QG_ERR_NULL otherwise). */
} qg_matrix_desc;

const char* qg_status_string(int status);
int qg_last_hip_error(void);

/* ---- Block-wise uniform quantization, Quant_n of Sec. 3.1 (z = 0, s = absmax/qmax,
 * code = clamp(round_half_even(fl32(x * fl32(qmax/absmax))), -2^(n-1), 2^(n-1)-1)).
 * A block whose absmax is 0 gets scale 0 and codes 0.
 * qg_quant_int8: x fp32 [rows][cols] -> q int8 [rows][cols], scales [rows][ceil(cols/256)].
 * qg_quant_int4: x fp32 [rows][cols] -> q_packed uint8 [ceil(rows*cols/2)], scales [ceil(rows*cols/256)].
 * Errors: NULL pointer, rows/cols <= 0 (or rows*cols >= 2^40), group, alignment. */
int qg_quant_int8(const float* x, int64_t rows, int64_t cols, int group,
                  int8_t* q, float* scales, void* stream);
int qg_quant_int4(const float* x, int64_t rows, int64_t cols, int group,
                  uint8_t* q_packed, float* scales, void* stream);

/* ---- Dequantization, W = W_q * s (Appendix A with zeros = 0); fp32 out [rows][cols]. */
int qg_dequant_int8(const int8_t* q, const float* scales, int64_t rows, int64_t cols, int group,
                    float* x, void* stream);
int qg_dequant_int4(const uint8_t* q_packed, const float* scales, int64_t rows, int64_t cols, int group,
                    float* x, void* stream);

/* ---- Gradient projection (Sec. 3.5): R = dequant(P)^T G.
 * P is dequantized inside the GEMM: code*scale in fp32, rounded once to bf16;
 * bf16 MFMA with fp32 accumulation; R fp32 [r][n] is overwritten.
 * Requires 1 <= r <= m, r % 8 == 0, m*n < 2^32.  `workspace` / `workspace_bytes`
 * are reserved: no kernel of this call uses scratch memory, the arguments are
 * not read and may be NULL / 0 (qg_workspace_bytes returns 0). */
int qg_project(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16,
               int64_t m, int64_t n, int64_t r, int group,
               float* R, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Adam on the low-rank gradient (Sec. 3.5; Adam of Sec. 4.1), element-wise over
 * count = r*n elements:  M <- b1 M + (1-b1) R;  V <- b2 V + (1-b2) R^2;
 * N = bf16( (M/(1-b1^t)) / (sqrt(V/(1-b2^t)) + eps) ).  M, V updated in place (fp32).
 * step = t >= 1.  R may not alias M, V or N. */
int qg_lowrank_adam(const float* R, float* M, float* V, uint16_t* N_bf16,
                    int64_t count, int64_t step, const qg_hparams* hp, void* stream);

/* ---- Adam with 8-bit states (Sec. 3.5: an 8-bit Adam is the paper's inner optimizer; it takes the state format from
 * a third-party library and does not define it - this format is this library's own design).
 * State format: block = 256 consecutive elements of the flattened r x n state; scales [ceil(count/256)] fp32 = the
 * block's absolute maximum; codes uint8 [count] = index of the entry nearest to x/scale (ties to the lower index) in
 * a sorted table with relative resolution.  Unsigned table (second moment): entry 0 is 0, entry p >= 1 has level
 * L = floor(log2 p), k = p - 2^L and value 10^-(7-L) * (0.1 + 0.9 (k+1) / 2^L) (2^L values spaced linearly over each
 * decade from 1e-7 to 1).  Signed table (first moment): levels 0..6 (1e-6 to 1), indices 0..126 the negatives from
 * -1 up, 127 zero, 128..254 the positives, 255 unused.  A positive second moment takes code 1 at least (it never
 * rounds to zero while the first moment, whose table reaches ten times further down, survives).
 * qg_state8_quant / qg_state8_dequant: fp32 [count] <-> (codes, scales); is_signed selects the table.
 * qg_lowrank_adam8: as qg_lowrank_adam, with M and V held in this format (Mq/Ms signed, Vq/Vs unsigned, updated in
 * place): dequantize (table[code] * scale), the same update and direction N, quantize again.
 * count >= 1, a multiple of 4, below 2^40; step >= 1. */
int qg_state8_quant(const float* x, int64_t count, int is_signed, uint8_t* codes, float* scales, void* stream);
int qg_state8_dequant(const uint8_t* codes, const float* scales, int64_t count, int is_signed, float* x, void* stream);
int qg_lowrank_adam8(const float* R, uint8_t* Mq, float* Ms, uint8_t* Vq, float* Vs, uint16_t* N_bf16,
                     int64_t count, int64_t step, const qg_hparams* hp, void* stream);
/* qg_step8: one full step on one matrix with 8-bit Adam states, the paper's default configuration (Sec. 3.5): qg_project
 * -> qg_lowrank_adam8 -> qg_backproject_update_sr on `stream`, with exactly their results.  R (fp32 r x n) and N are
 * caller-provided scratch outputs and both required. */
int qg_step8(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16, int8_t* Wq, float* Ws,
             uint8_t* Mq, float* Ms, uint8_t* Vq, float* Vs, float* R, uint16_t* N_bf16,
             int64_t m, int64_t n, int64_t r, int group, const qg_hparams* hp, uint64_t seed, int64_t step, void* stream);

/* ---- Projection and Adam fused (Sec. 3.5): the same arithmetic as qg_project followed by qg_lowrank_adam, with
 * Adam applied in the GEMM epilogue while R is still in registers.  M, V in/out, N out; R (nullable) receives the
 * projected gradient only if the caller wants to inspect it - leaving it NULL saves writing and re-reading
 * 8 bytes per low-rank element.  Results are bit-identical to the two separate calls.  This is the form qg_step
 * and qg_step_many run. */
int qg_project_adam(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16,
                    float* R /* nullable */, float* M, float* V, uint16_t* N_bf16,
                    int64_t m, int64_t n, int64_t r, int group, int64_t step, const qg_hparams* hp, void* stream);

/* ---- Back-projection and INT8 weight update with stochastic rounding
 * (Sec. 3.4, Sec. 3.5):  U = alpha * dequant(P) * N;  x = W_q*s - lr*U;  per block
 * of 256 of each row a = max|x|, s' = a/127, code' = clamp(floor(x*(127/a) + u), -128, 127)
 * with u = 2^-24 * (hash32(seed, step, i*n+j) >> 8).  Wq and Ws are updated in
 * place.  U_debug (nullable) receives U as fp32 [m][n] for parity checks.
 * Requires r % 8 == 0, r <= m, m*n < 2^32. */
int qg_backproject_update_sr(const uint8_t* Pq, const float* Ps, const uint16_t* N_bf16,
                             int8_t* Wq, float* Ws, int64_t m, int64_t n, int64_t r, int group,
                             float alpha, float lr, uint64_t seed, int64_t step,
                             float* U_debug, void* stream);

/* ---- Subspace convergence check (Sec. 3.2, Fig. 2): mean over the r columns of
 * the cosine between column k of dequant(PA) and of dequant(PB).  cos_out is one
 * device float.  workspace: at least qg_cossim_workspace_bytes(m, r) bytes. */
size_t qg_cossim_workspace_bytes(int64_t m, int64_t r);
int qg_subspace_cossim(const uint8_t* PqA, const float* PsA, const uint8_t* PqB, const float* PsB,
                       int64_t m, int64_t r, int group, float* cos_out,
                       void* workspace, size_t workspace_bytes, void* stream);

/* qg_subspace_cossim_weighted: sum_k w_k cos_k / sum_k w_k over the same column cosines, with non-negative weights
 * w (device, fp32 [r], 4-byte aligned; NULL = the plain mean above).  The subspace refresh below reports this form,
 * with the gradient energy each new column captures as the weights.  Same workspace and errors. */
int qg_subspace_cossim_weighted(const uint8_t* PqA, const float* PsA, const uint8_t* PqB, const float* PsB,
                                const float* weights, int64_t m, int64_t r, int group, float* cos_out,
                                void* workspace, size_t workspace_bytes, void* stream);

/* ---- qg_subspace_cossim for callers that cannot allocate device memory or carry a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same kernels and the same result, with the
 * partial sums in a 4 MiB device array that is part of the library image (each GPU that loads the library holds its
 * own copy until the process ends).  Limit: qg_cossim_workspace_bytes(m, r) <= 4 MiB, i.e. about
 * ceil(m/64) * 3 * r <= 2^20 (m = 11008 with r = 1024 fits); larger shapes return QG_ERR_WORKSPACE.  The call
 * allocates nothing and frees nothing; its first call on a device looks the array's address up (make that call
 * outside graph capture).  All calls on one GPU share the array: calls that overlap on one GPU (different streams
 * or threads) race; calls on one stream are ordered and safe.  Other errors as qg_subspace_cossim. */
int qg_subspace_cossim_static(const uint8_t* PqA, const float* PsA, const uint8_t* PqB, const float* PsB,
                              int64_t m, int64_t r, int group, float* cos_out, void* stream);

/* ---- Subspace refresh (Sec. 3.2: every `interval` steps the projection is recomputed from the current gradient;
 * the paper takes the first r left singular vectors of G).  One pass of orthogonal iteration started from the stored
 * projection stands in for the SVD; it converges to the same singular vectors, in the same order, at the rate
 * (sigma_{r+1} / sigma_r)^2 per pass:
 *     R = dequant(P)^T G (qg_project);  Z = bf16(R);  Y = G Z^T;  Q = orthonormalize(Y);  P_new = quant_int4(Q)
 * and, after the last pass, the convergence check of Sec. 3.2 between P and P_new:
 *     *cos_out = qg_subspace_cossim_weighted(P, P_new, e),   e_k = sum_j (dequant(P_new)^T G)[k][j]^2,
 * the column cosines weighted with the gradient energy each new column captures.  (The iteration starts from the old
 * projection, so columns that capture next to no energy come back much as they went in whatever the gradient does;
 * unweighted they would dominate the mean.  With comparable energies in all columns it is the plain mean.)
 *
 * qg_range_apply: Y (fp32 [m][r], overwritten) = G (bf16 [m][n]) * Z^T (Z bf16 [r][n]); bf16 MFMA, fp32 accumulation.
 *
 * qg_orthonormalize: Q (fp32 [m][r]) = the orthonormal factor of Y = Q T with T upper triangular and a positive
 * diagonal (Gram-Schmidt on the columns of Y in order), computed in fp64 as Q = Y L^-T from the Cholesky factor
 * of Y^T Y, twice in a row (the second round removes the cond(Y)^2 loss of orthogonality of the first; accurate to
 * fp32 rounding of what Householder QR gives for cond(Y) up to several 1e8; a shift of 2^-46 trace(Y^T Y) on the
 * Gram diagonal keeps the pivots positive).  *info (device int32) receives 0, or 1 + the index of the first column
 * found numerically dependent on its predecessors (Y rank deficient: that column of Q and the later ones are then
 * meaningless, but every kernel still completes).  Y and Q may not alias.
 * workspace: qg_orthonormalize_workspace_bytes(m, r) bytes, 16-byte aligned.
 *
 * qg_subspace_refresh_many: `passes` (1 .. 64) passes as above on `count` matrices of ONE shape (m, n, r).  descs
 * is a HOST array; Pq/Ps hold each matrix's old projection (unchanged), Pq_new/Ps_new (same sizes, distinct
 * buffers) receive the new one.  cos_out and info are device arrays of `count` elements (info as for
 * qg_orthonormalize, first failure over all passes).  The fp64 stages run batched over the matrices, as many at a
 * time as the workspace holds: qg_refresh_workspace_bytes(count, m, n, r) bytes let all of them run in one batch,
 * qg_refresh_workspace_bytes(1, m, n, r) is the minimum; results do not depend on the batch size.  workspace is
 * 16-byte aligned; after the call it starts with dequant(P_new)^T G (fp32 [r][n]) of the last matrix.
 * qg_subspace_refresh: the same for one matrix.
 * qg_subspace_refresh_many_ld: the same with gradients stored at a row pitch of ld elements (ld >= n, a multiple of
 * 16, or ld == n / 0 for dense rows; m*ld and r*ld below 2^32): rows then start 16-byte aligned whatever n is (the
 * 2048 x 5461 matrices of the LLaMA-1B shapes).  Size the workspace with qg_refresh_workspace_bytes(count, m, ld, r).
 *
 * All require r % 8 == 0, r <= m, m*r < 2^31 and m*n < 2^32 (QG_ERR_SHAPE otherwise). */
typedef struct {
    const uint8_t*  Pq;      /* old projection, INT4 packed  */
    const float*    Ps;      /* old projection, block scales */
    const uint16_t* G;       /* bf16 gradient m x n          */
    uint8_t*        Pq_new;  /* out */
    float*          Ps_new;  /* out */
} qg_refresh_desc;
int qg_range_apply(const uint16_t* G_bf16, const uint16_t* Z_bf16, int64_t m, int64_t n, int64_t r, float* Y,
                   void* stream);
size_t qg_orthonormalize_workspace_bytes(int64_t m, int64_t r);
int qg_orthonormalize(const float* Y, int64_t m, int64_t r, float* Q, int32_t* info,
                      void* workspace, size_t workspace_bytes, void* stream);
size_t qg_refresh_workspace_bytes(int count, int64_t m, int64_t n, int64_t r);
int qg_subspace_refresh_many(int count, const qg_refresh_desc* descs, int64_t m, int64_t n, int64_t r, int group,
                             int passes, float* cos_out, int32_t* info,
                             void* workspace, size_t workspace_bytes, void* stream);
int qg_subspace_refresh_many_ld(int count, const qg_refresh_desc* descs, int64_t m, int64_t n, int64_t ld, int64_t r,
                                int group, int passes, float* cos_out, int32_t* info,
                                void* workspace, size_t workspace_bytes, void* stream);
int qg_subspace_refresh(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16,
                        int64_t m, int64_t n, int64_t r, int group, int passes,
                        uint8_t* Pq_new, float* Ps_new, float* cos_out, int32_t* info,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---- INT8 linear layer (Appendix A): the layer whose weight the step updates; its backward pass produces the
 * gradient G the step consumes.  W is the m x n INT8 weight (codes + block scales as above, zero point 0),
 * dequantized inside the GEMMs as bf16(fl32(code * scale)); bf16 MFMA, fp32 accumulation, outputs rounded once
 * to bf16 (activations and gradients are BFloat16, Sec. 3.1).
 * qg_int8_linear_forward:  y [tokens][m] = x [tokens][n] * W^T (+ bias [m], bf16, nullable).
 * qg_int8_linear_backward: dx [tokens][n] = dy [tokens][m] * W and G [m][n] = dy^T * x; either output may be NULL
 *   (then it is not computed, and the inputs only it needs - Wq/Ws for dx, x for G - may be NULL too).
 * Any tokens, m, n >= 1 with tokens*m, tokens*n and m*n below 2^31; base pointers 16-byte aligned (rows need not
 * be).  Outputs may not alias inputs. */
int qg_int8_linear_forward(const uint16_t* x_bf16, const int8_t* Wq, const float* Ws, const uint16_t* bias_bf16,
                           int64_t tokens, int64_t m, int64_t n, int group, uint16_t* y_bf16, void* stream);
int qg_int8_linear_backward(const uint16_t* dy_bf16, const uint16_t* x_bf16, const int8_t* Wq, const float* Ws,
                            int64_t tokens, int64_t m, int64_t n, int group,
                            uint16_t* dx_bf16, uint16_t* G_bf16, void* stream);

/* The same two calls on arrays stored at a row pitch: ld_n is the pitch of the arrays with n elements per row (x, dx,
 * Wq, G), ld_m that of the arrays with m (y, dy); each is the row length itself (or 0), or at least it and a multiple
 * of 16 elements, with rows * pitch below 2^31.  Rows then start 16-byte aligned whatever m and n are (n = 5461 in the
 * LLaMA-1B shapes); G comes out in the layout qg_step_ld and the `ld` of qg_matrix_desc take.  Scales stay
 * [m][ceil(n/256)].  Padding is never read for a result and never written. */
int qg_int8_linear_forward_ld(const uint16_t* x_bf16, const int8_t* Wq, const float* Ws, const uint16_t* bias_bf16,
                              int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group,
                              uint16_t* y_bf16, void* stream);
int qg_int8_linear_backward_ld(const uint16_t* dy_bf16, const uint16_t* x_bf16, const int8_t* Wq, const float* Ws,
                               int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group,
                               uint16_t* dx_bf16, uint16_t* G_bf16, void* stream);

/* ---- Right-side projection (GaLore's second form, which Sec. 3.5 inherits: R = G Q with Q the n x r matrix of right
 * singular vectors, moments m x r, update alpha N Q^T; used where a weight has more rows than columns).  A weight
 * that is projected from the right is kept TRANSPOSED, S = W^T: n x m INT8 codes, blocks of 256 along each row of S,
 * scales [n][ceil(m/256)].  Its optimizer step, subspace refresh and cosine check are then the left-side calls above
 * on the n x m matrix S with P = Q (n x r) and the gradient in S's layout: qg_step(Qq, Qs, G_S, Sq, Ss, M, V, R, N,
 * n, m, r, ...) with moments r x m (the transposes of GaLore's m x r; Adam is element-wise).  The two calls below are
 * the linear layer on that storage; its backward pass writes the gradient directly in S's layout, so nothing is ever
 * transposed in memory.
 * qg_int8_linear_t_forward:  y [tokens][m] = x [tokens][n] * S (+ bias [m], bf16, nullable)      (= x W^T)
 * qg_int8_linear_t_backward: dx [tokens][n] = dy [tokens][m] * S^T                                (= dy W)
 *                            G_S [n][m] = x^T * dy                                               (= (dy^T x)^T)
 * Arguments, limits, NULL outputs and alignment as for the two calls above. */
int qg_int8_linear_t_forward(const uint16_t* x_bf16, const int8_t* Sq, const float* Ss, const uint16_t* bias_bf16,
                             int64_t tokens, int64_t m, int64_t n, int group, uint16_t* y_bf16, void* stream);
int qg_int8_linear_t_backward(const uint16_t* dy_bf16, const uint16_t* x_bf16, const int8_t* Sq, const float* Ss,
                              int64_t tokens, int64_t m, int64_t n, int group,
                              uint16_t* dx_bf16, uint16_t* GS_bf16, void* stream);

/* ---- Zero-point (asymmetric) INT8 weights: the quantizer as Sec. 3.1 writes it, W_q = clamp(round(W/s) + z), and
 * Appendix A's dequantization W = (W_q - zeros) * scales.  Per block of 256 elements of a row: lo = min(0, min x),
 * hi = max(0, max x), s = (hi - lo)/255, z = clamp(-128 - round(lo * (255/(hi - lo))), -128, 127), code =
 * clamp(round(x * (255/(hi - lo))) + z, -128, 127), all in fp32; an all-zero block has s = 0, z = 0.  Zero points are
 * whole numbers kept as fp32 [rows][ceil(cols/256)], next to the scales.  Zero itself is always a code (z).
 * qg_quant_int8_zp / qg_dequant_int8_zp: as qg_quant_int8 / qg_dequant_int8, with the zero points.
 * qg_backproject_update_sr_zp: as qg_backproject_update_sr on such a weight: x = (W_q - z)*s - lr*U, new (s', z')
 *   from the block's min and max as above, code' = clamp(floor(x*(255/(hi - lo)) + u) + z', -128, 127) with the same
 *   uniform draw u; Wq, Ws, Wz updated in place.
 * qg_step_zp: qg_step on such a weight (qg_project_adam, then qg_backproject_update_sr_zp); in a grouped plan give
 *   every descriptor its Wz.
 * qg_int8_linear_zp_forward / _backward: the linear layer on such a weight (W dequantized inside the GEMMs as
 *   bf16(fl32((code - zero) * scale))).
 * qg_int8_linear_t_zp_forward / _backward: the same on a zero-point weight stored transposed (S = W^T: codes
 *   [n][m], scales and zero points [n][ceil(m/256)]), the layer of a right-projected matrix in this format; its
 *   step is qg_step_zp on S as for the symmetric format.
 * Shapes, limits, alignment and NULL rules as for the calls they mirror; Wz may never be NULL. */
int qg_quant_int8_zp(const float* x, int64_t rows, int64_t cols, int group, int8_t* q, float* scales, float* zeros,
                     void* stream);
int qg_dequant_int8_zp(const int8_t* q, const float* scales, const float* zeros, int64_t rows, int64_t cols, int group,
                       float* x, void* stream);
int qg_backproject_update_sr_zp(const uint8_t* Pq, const float* Ps, const uint16_t* N_bf16,
                                int8_t* Wq, float* Ws, float* Wz, int64_t m, int64_t n, int64_t r, int group,
                                float alpha, float lr, uint64_t seed, int64_t step, void* stream);
int qg_step_zp(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16,
               int8_t* Wq, float* Ws, float* Wz, float* M, float* V, float* R, uint16_t* N_bf16,
               int64_t m, int64_t n, int64_t r, int group,
               const qg_hparams* hp, uint64_t seed, int64_t step, void* stream);
int qg_int8_linear_zp_forward(const uint16_t* x_bf16, const int8_t* Wq, const float* Ws, const float* Wz,
                              const uint16_t* bias_bf16, int64_t tokens, int64_t m, int64_t n, int group,
                              uint16_t* y_bf16, void* stream);
int qg_int8_linear_zp_backward(const uint16_t* dy_bf16, const uint16_t* x_bf16, const int8_t* Wq, const float* Ws,
                               const float* Wz, int64_t tokens, int64_t m, int64_t n, int group,
                               uint16_t* dx_bf16, uint16_t* G_bf16, void* stream);
int qg_int8_linear_t_zp_forward(const uint16_t* x_bf16, const int8_t* Sq, const float* Ss, const float* Sz,
                                const uint16_t* bias_bf16, int64_t tokens, int64_t m, int64_t n, int group,
                                uint16_t* y_bf16, void* stream);
int qg_int8_linear_t_zp_backward(const uint16_t* dy_bf16, const uint16_t* x_bf16, const int8_t* Sq, const float* Ss,
                                 const float* Sz, int64_t tokens, int64_t m, int64_t n, int group,
                                 uint16_t* dx_bf16, uint16_t* GS_bf16, void* stream);

/* ---- Residual stream between two blocks of a decoder: the norm behind a block, its gate and residual scale, the sum,
 * and the norm ahead of the next block, in one pass.  For each of `tokens` rows of d elements, rms(v) = sqrt(mean v^2 + eps):
 *     n  = w_post * y / rms(y)            y: the block's output, bf16; w_post NULL: n = y
 *     h' = h + scale * gate * n           gate_kind: none (1), fp32 [d], or bf16 [tokens][ld]
 *     u  = w_pre * h' / rms(h')           bf16; from h' as it is before it is rounded to the stream's type
 * h and h' (h_out) are bf16, or fp32 with stream_fp32 != 0.  y NULL: h' = h, h_out is not written (a norm alone).
 * u NULL: not computed.  h_out may be h.  w_post, w_pre: fp32 [d].  eps: 0 or more (with 0, a row of zeros has no rms).
 *
 * qg_residual_norm_backward: the gradients at h_next = h' as stored, given du and dh_next (the stream's own gradient at
 * h', in the stream's type; either may be NULL: 0): dh of h and, in the sum, of h' alike (may be dh_next), dy (bf16),
 * dw_pre, dw_post (fp32 [d]) and dgate (fp32 [d], or bf16 [tokens][ld]); dw_pre, dw_post and dgate are each optional.  y
 * NULL: no block output, only dh and dw_pre.  rms is computed again from h_next and y.  Sums over tokens are added in a
 * fixed order.  workspace: qg_residual_norm_workspace_bytes(tokens, d) bytes, 16-byte aligned; may be NULL / 0 if none of
 * dw_pre, dw_post and a channel's dgate is asked for.
 *
 * tokens below 2^22, 1 <= d <= 16384.  ld: row pitch of every [tokens][d] array: d (or 0), or more and a multiple of 16;
 * padding is neither read nor written. */
enum { QG_GATE_NONE = 0, QG_GATE_CHANNEL = 1, QG_GATE_TOKEN = 2 };
int qg_residual_norm_forward(const void* h, const uint16_t* y_bf16, const float* w_post, const void* gate, int gate_kind,
                             const float* w_pre, float scale, float eps, int64_t tokens, int64_t d, int64_t ld, int stream_fp32,
                             void* h_out, uint16_t* u_bf16, void* stream);
size_t qg_residual_norm_workspace_bytes(int64_t tokens, int64_t d);
int qg_residual_norm_backward(const uint16_t* du_bf16, const void* dh_next, const void* h_next, const uint16_t* y_bf16,
                              const float* w_post, const void* gate, int gate_kind, const float* w_pre, float scale, float eps,
                              int64_t tokens, int64_t d, int64_t ld, int stream_fp32, void* dh, uint16_t* dy_bf16,
                              float* dw_pre, float* dw_post, void* dgate, void* workspace, size_t workspace_bytes, void* stream);

/* ---- INT8 linear layer with an epilogue, and the gated pair of a feed-forward block.  Weights, dequantization, pitches and
 * limits as for qg_int8_linear_forward_ld (ld_n: x, dx, W, G; ld_m: y, z, residual, dy, dz; 0: dense).
 * act: one of QG_ACT_*; silu(z) = z / (1 + exp(-z)), gelu(z) = z Phi(z) with the normal distribution's cdf.
 *
 * qg_int8_linear_act_forward:  z = x W^T + bias (bf16 [m], nullable);  y = act(z) + residual (bf16 [tokens][ld_m], nullable).  The
 *   activation takes the fp32 sum; z (nullable) is what the backward pass wants, rounded to bf16.  y may be residual.
 * qg_int8_linear_act_backward: dz = dy act'(z);  dx = dz W, G = dz^T x, dbias (fp32 [m]) = sum over tokens of dz, each of them
 *   nullable (and then the inputs only it needs are too).  dz is rounded to bf16 for the products, not for dbias.  QG_ACT_NONE
 *   needs no z.  The residual's gradient is dy.  workspace: qg_int8_linear_act_workspace_bytes(tokens, m, n) bytes, 16-byte aligned;
 *   not needed for dx and G with QG_ACT_NONE.
 * qg_int8_gated_forward:  y = act(x Wg^T) * (x Wu^T), both weights m x n; zg, zu: both (for the backward pass) or neither.
 * qg_int8_gated_backward: dzg = dy zu act'(zg), dzu = dy act(zg), rounded to bf16;  dx = dzg Wg + dzu Wu (nullable), Gg = dzg^T x
 *   and Gu = dzu^T x (both or neither).  workspace: qg_int8_gated_workspace_bytes(tokens, m, n) bytes, 16-byte aligned. */
enum { QG_ACT_NONE = 0, QG_ACT_RELU = 1, QG_ACT_SILU = 2, QG_ACT_GELU = 3 };
int qg_int8_linear_act_forward(const uint16_t* x_bf16, const int8_t* Wq, const float* Ws, const uint16_t* bias_bf16,
                               const uint16_t* residual_bf16, int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n,
                               int64_t ld_m, int group, uint16_t* z_bf16, uint16_t* y_bf16, void* stream);
size_t qg_int8_linear_act_workspace_bytes(int64_t tokens, int64_t m, int64_t n);
int qg_int8_linear_act_backward(const uint16_t* dy_bf16, const uint16_t* z_bf16, const uint16_t* x_bf16, const int8_t* Wq,
                                const float* Ws, int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group,
                                uint16_t* dx_bf16, uint16_t* G_bf16, float* dbias, void* workspace, size_t workspace_bytes,
                                void* stream);
int qg_int8_gated_forward(const uint16_t* x_bf16, const int8_t* Wgq, const float* Wgs, const int8_t* Wuq, const float* Wus, int act,
                          int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group, uint16_t* zg_bf16,
                          uint16_t* zu_bf16, uint16_t* y_bf16, void* stream);
size_t qg_int8_gated_workspace_bytes(int64_t tokens, int64_t m, int64_t n);
int qg_int8_gated_backward(const uint16_t* dy_bf16, const uint16_t* zg_bf16, const uint16_t* zu_bf16, const uint16_t* x_bf16,
                           const int8_t* Wgq, const float* Wgs, const int8_t* Wuq, const float* Wus, int act, int64_t tokens,
                           int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group, uint16_t* dx_bf16, uint16_t* Gg_bf16,
                           uint16_t* Gu_bf16, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Loss of a language model's head: softmax cross entropy over the vocabulary, without the logits in memory.
 * z = x W^T with x bf16 [tokens][h] and W bf16 [vocab][h]; labels int64 [tokens], a label outside [0, vocab) marks a token
 * without a loss (padding, a prompt): its loss, lse and row of dx are 0, and it adds nothing to dW whatever its row of x holds.
 * Such tokens take no part in the products; what that saves comes in steps of 64 to 256 tokens, and is least in dx of a batch of
 * thousands with few labels.
 * qg_head_loss_forward:  lse = log sum_v exp z_v, loss = lse - z_label, fp32 [tokens].
 * qg_head_loss_backward: from lse and dloss (fp32 [tokens], the gradient of each token's loss: a mean's 1/count, a weight),
 *   dz = dloss (exp(z - lse) - onehot), rounded to bf16;  dx = dz W, dW = dz^T x, either may be NULL.  The vocabulary is
 *   taken in pieces: the logits of a piece are computed again, and only tokens x piece numbers are stored.
 * ld: row pitch of x, W, dx and dW: h (or 0), or more and a multiple of 16.  tokens and vocab below 2^24, h below 2^16,
 * tokens * vocab below 2^38, tokens * h below 2^34, vocab * h below 2^37.  workspace: qg_head_loss_workspace_bytes(tokens, h, vocab) bytes, 16-byte
 * aligned, enough for either call.  labels need 8-byte alignment only, loss, lse and dloss 4-byte (views shifted by a token). */
size_t qg_head_loss_workspace_bytes(int64_t tokens, int64_t h, int64_t vocab);
int qg_head_loss_forward(const uint16_t* x_bf16, const uint16_t* W_bf16, const int64_t* labels, int64_t tokens, int64_t h,
                         int64_t vocab, int64_t ld, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream);
int qg_head_loss_backward(const uint16_t* x_bf16, const uint16_t* W_bf16, const int64_t* labels, const float* lse,
                          const float* dloss, int64_t tokens, int64_t h, int64_t vocab, int64_t ld, uint16_t* dx_bf16,
                          uint16_t* dW_bf16, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Attention half of a decoder layer: rotary positions, attention over packed sequences, and a cache of keys and values in pages with
 * the attention of one new token over it.
 *
 * qg_heads: a bf16 array [tokens][heads][d] with the strides given, in elements, both multiples of 8, token_stride below 2^23
 *   (so that q, k and v may be slices of one linear layer's output, or heads may be the outer index).  Elements of a head are consecutive.
 *
 * qg_rope_forward: the pairs (a, b) of the first `rot` elements of every head of q and k (k may be NULL, with heads_k = 0) become
 *     amplitude * (a cos t - b sin t, a sin t + b cos t),   t = positions[token] * freqs[pair];
 *   QG_ROPE_HALF: pair i is elements (i, i + rot/2), QG_ROPE_INTERLEAVED: (2i, 2i + 1); elements from rot on are copied.  rot is even, 2 <= rot <= d;
 *   1 <= d <= 1024, and where d is no multiple of 8 strides may be any and data 2-byte aligned; positions int64, freqs double [rot/2] (device).  Angles are formed in 64 bits.  An output may be its input,
 *   and overlap neither an input nor an output otherwise.  tokens below 2^24, heads up to 1024.
 * qg_rope_backward: its gradients, turned back: dq and dk from those of the outputs (the same call with -t).
 * qg_rope_frequencies (HOST ONLY, `out` is a host pointer to rot/2 doubles): base^(-2i/rot); with a factor other than 1 stretched to longer
 *   contexts: frequencies that turn at most `low` times over `context` positions are divided by factor, those that turn at least `high`
 *   times are kept, those between go from one to the other linearly in their turns; context 0: all are divided.
 *
 * qg_attention_forward: for each query of a sequence, over the keys of the same sequence that are visible to it,
 *     x = scale q.k;  cap > 0: x = cap tanh(x / cap);  slopes: x -= slopes[head] |distance|;  o = softmax(x) v, lse = log sum exp x.
 *   Tokens are packed: sequence i has queries cu_q[i] .. cu_q[i+1] - 1 and keys cu_k[i] .. cu_k[i+1] - 1 (int32 [sequences + 1] on the device,
 *   ascending, the first is 0; cu_k NULL: the queries' (tokens_q = tokens_k then); both NULL: one sequence of all tokens).  Query i of a
 *   sequence stands at position i + n_keys - n_queries, the distance to key j is that minus j.  Visible: with causal, keys that are not
 *   behind the query and, with window > 0, nearer than window, or, with prefix (int32 [sequences]), among the first prefix keys of the
 *   sequence; window and prefix exclude each other and need causal; without causal all keys.  Query head h reads key head
 *   h / (heads_q / heads_k).  lse: fp32 [heads_q][tokens_q], may be NULL.  A query without a visible key, and tokens behind
 *   the last sequence: o = 0, lse = -inf.  Those tokens' q, k and v are not read; inside a sequence a value that is not finite can
 *   reach every query of its sequence, and every gradient.
 * qg_attention_backward: dq, dk, dv from do, the forward pass's inputs and its o and lse (delta = sum do o from o as
 *   stored, corrected by what the sum of the scores' gradients over a row, which is 0, then comes to).  Sums of the heads that
 *   share k and v, and over tokens, are added in a fixed order.  Slopes have no gradient.
 *   d: a multiple of 8 up to 128.  scale, and a cap that is not 0, from 2^-60 to 2^60.  No output may overlap an input or another output.  tokens below 2^24, heads up to 1024, sequences up to 2^20, tokens * heads below 2^30, sequences * heads below 2^23.
 *   workspace: qg_attention_forward_workspace_bytes(a) or qg_attention_backward_workspace_bytes(a) bytes, 16-byte aligned; NULL where that is 0;
 *   calls that may run at the same time need one each.
 *
 * qg_cache: keys and values of `sequences` sequences in pages: position p of sequence s is row p % page_size of page
 *   table[s][p / page_size].  An entry outside [0, pages) has no page: nothing is written there, and its keys are not visible.
 *   pages * page_size and sequences * width below 2^31, width * page_size below 2^30, heads up to 1024, sequences up to 2^20, 8 <= d <= 1024 and a
 *   multiple of 8.
 * qg_cache_append: k and v of `tokens` tokens to their place: token t belongs to sequence[t] (NULL: t) and stands at positions[t]; one without
 *   a place is left out.  k is turned as by qg_rope_forward on its way, and so is q (NULL, with heads_q = 0: none) to q_out (may be q); rot 0:
 *   nothing is turned (freqs NULL).  Tokens of one call need places of
 *   their own: one that two of them share ends up with pieces of both.  The pages of k and v, and q_out, may not overlap each other, and no place that
 *   is written may hold an input of the call (but q_out q).
 * qg_attention_paged: one new token per sequence: o = softmax over positions 0 .. lengths[s] - 1 of the cache, the query standing
 *   at lengths[s] - 1 (a length beyond width * page_size counts as that); scores, scale, cap, slopes and window as above; d up to 128, sequences * heads_q below 2^24.  No length (or no page): o = 0.  o may be q, and
 *   overlap no input otherwise.  What the
 *   cache holds outside the visible positions is not looked at.  workspace: qg_attention_paged_workspace_bytes(c, heads_q) bytes, 16-byte
 *   aligned; calls that may run at the same time need one each. */
typedef struct {
    uint16_t* data;
    int64_t token_stride, head_stride;
} qg_heads;
enum { QG_ROPE_HALF = 0, QG_ROPE_INTERLEAVED = 1 };
int qg_rope_frequencies(int rot, double base, double factor, double context, double low, double high, double* out);
int qg_rope_forward(const qg_heads* q, int heads_q, const qg_heads* k, int heads_k, const int64_t* positions, const double* freqs,
                    int64_t tokens, int d, int rot, int layout, float amplitude, const qg_heads* q_out, const qg_heads* k_out, void* stream);
int qg_rope_backward(const qg_heads* dq_out, int heads_q, const qg_heads* dk_out, int heads_k, const int64_t* positions, const double* freqs,
                     int64_t tokens, int d, int rot, int layout, float amplitude, const qg_heads* dq, const qg_heads* dk, void* stream);

typedef struct {
    int64_t tokens_q, tokens_k;         /* rows of q and o, of k and v */
    int heads_q, heads_k, d, sequences;
    const int32_t *cu_q, *cu_k;
    const int32_t* prefix;
    const float* slopes;
    float scale, cap;
    int causal;
    int64_t window;
} qg_attention;
size_t qg_attention_forward_workspace_bytes(const qg_attention* a);
size_t qg_attention_backward_workspace_bytes(const qg_attention* a);
int qg_attention_forward(const qg_attention* a, const qg_heads* q, const qg_heads* k, const qg_heads* v, const qg_heads* o, float* lse,
                         void* workspace, size_t workspace_bytes, void* stream);
int qg_attention_backward(const qg_attention* a, const qg_heads* dO, const qg_heads* q, const qg_heads* k, const qg_heads* v,
                          const qg_heads* o, const float* lse, const qg_heads* dq, const qg_heads* dk, const qg_heads* dv, void* workspace,
                          size_t workspace_bytes, void* stream);

typedef struct {
    uint16_t *k, *v;                    /* [pages][page_size][heads][d] each, 16-byte aligned */
    const int32_t* table;               /* [sequences][width] */
    int64_t pages;
    int page_size, heads, d, sequences, width;
} qg_cache;
int qg_cache_append(const qg_cache* c, const qg_heads* q, int heads_q, const qg_heads* k, const qg_heads* v, const int64_t* positions,
                    const int32_t* sequence, int64_t tokens, const double* freqs, int rot, int layout, float amplitude,
                    const qg_heads* q_out, void* stream);
size_t qg_attention_paged_workspace_bytes(const qg_cache* c, int heads_q);
int qg_attention_paged(const qg_cache* c, const int32_t* lengths, const qg_heads* q, int heads_q, float scale, float cap, int64_t window,
                       const float* slopes, const qg_heads* o, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Adaptive lazy update policy (Sec. 3.2), HOST ONLY (p is a host pointer):
 * streak counts consecutive checks with cos >= threshold; at k in a row the
 * interval doubles and the streak restarts; next_refresh advances by the
 * (possibly doubled) interval.  Returns 1 if the interval doubled, 0 if not,
 * -1 if p is NULL. */
int qg_policy_update(qg_policy* p, float cos);

/* ---- One full step on one matrix (Sec. 3.5): project -> Adam -> back-project +
 * SR update, as two kernels on `stream` (qg_project_adam, then
 * qg_backproject_update_sr): the same results as the three separate calls.
 * N is a caller-provided output (r x n bf16); R (r x n fp32) is written only
 * if it is not NULL.  No subspace refresh happens inside.
 * qg_workspace_bytes: scratch bytes qg_project and qg_step need for a matrix of
 * this shape: always 0 (both run out of registers and LDS); their `workspace`
 * and `workspace_bytes` arguments are reserved, never read, and may be NULL / 0. */
size_t qg_workspace_bytes(int64_t m, int64_t n, int64_t r);
int qg_step(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16,
            int8_t* Wq, float* Ws, float* M, float* V, float* R, uint16_t* N_bf16,
            int64_t m, int64_t n, int64_t r, int group,
            const qg_hparams* hp, uint64_t seed, int64_t step,
            void* workspace, size_t workspace_bytes, void* stream);

/* qg_step_ld: qg_step on arrays stored at a row pitch: G, Wq (m rows) and M, V, R, N (r rows) all have rows ld
 * elements apart (ld >= n and a multiple of 16, or ld == n / 0 for dense rows; m*ld < 2^32), as in the `ld` field of
 * qg_matrix_desc: a matrix whose n is not a multiple of 8 then runs in the kernels for 16-byte aligned rows.  Scales
 * stay [m][ceil(n/256)]; the stochastic-rounding index stays i*n + j, so the n real columns get the dense layout's
 * result.  Padding is never read for a result and not written. */
int qg_step_ld(const uint8_t* Pq, const float* Ps, const uint16_t* G_bf16,
               int8_t* Wq, float* Ws, float* M, float* V, float* R, uint16_t* N_bf16,
               int64_t m, int64_t n, int64_t ld, int64_t r, int group,
               const qg_hparams* hp, uint64_t seed, int64_t step, void* stream);

/* ---- Grouped step over many matrices (the whole model's linear weights) in
 * two grouped launches per edge class (projection with Adam in its epilogue,
 * back-projection + update).  R is written only if every descriptor supplies
 * a buffer for it; qg_project_many and qg_lowrank_adam_many need every R.
 * `descs` is a HOST array of `count` descriptors.
 * The library needs a device-resident launch plan: the caller provides
 * `plan_host` (host scratch) and `plan_dev` (device memory), each of
 * qg_plan_bytes(count, descs) bytes; qg_plan_build fills plan_host, the
 * caller copies it to plan_dev (any memcpy), and qg_step_many uses both.
 * Matrix i draws its SR numbers with seed + i * 0x9E3779B97F4A7C15 (mod 2^64). */
size_t qg_plan_bytes(int count, const qg_matrix_desc* descs);
int qg_plan_build(int count, const qg_matrix_desc* descs, void* plan_host, size_t plan_bytes);
int qg_step_many(int count, const void* plan_host, const void* plan_dev, size_t plan_bytes,
                 const qg_hparams* hp, uint64_t seed, int64_t step, void* stream);

/* The grouped launches one by one (same plan arguments): projection of every matrix, Adam over every matrix
 * (these two need every descriptor's R), their fusion (write_R != 0 also stores R), and back-projection + SR update
 * of every matrix.  qg_step_many(...) == qg_project_adam_many, qg_backproject_update_sr_many; the unfused pair
 * qg_project_many, qg_lowrank_adam_many gives bit-identical M, V, N (and R). */
int qg_project_many(int count, const void* plan_host, const void* plan_dev, size_t plan_bytes, void* stream);
int qg_lowrank_adam_many(int count, const void* plan_host, const void* plan_dev, size_t plan_bytes,
                         const qg_hparams* hp, int64_t step, void* stream);
int qg_project_adam_many(int count, const void* plan_host, const void* plan_dev, size_t plan_bytes,
                         const qg_hparams* hp, int64_t step, int write_R, void* stream);
int qg_backproject_update_sr_many(int count, const void* plan_host, const void* plan_dev, size_t plan_bytes,
                                  const qg_hparams* hp, uint64_t seed, int64_t step, void* stream);

/* ---- Measurement helpers (no part of the method; used by the benchmark to state what the machine sustains).
 *
 * qg_diag_clock_probe: enqueues a one-wave kernel that waits ticks_100mhz ticks (1 .. 10^8) of the constant
 * 100 MHz counter and writes {shader clock cycles elapsed, ticks elapsed} to out2 (device, 2 x int64).  Launched
 * on a second stream beside a kernel under test it gives the shader clock that kernel runs at.
 *
 * qg_diag_mfma_loop: QG_DIAG_MFMA_WORKGROUPS workgroups of 512 threads (8 waves, two per SIMD); each wave issues
 * iters (1 .. 2^24) rounds of 16 independent bf16 32x32x16 MFMAs on register operands, i.e.
 * QG_DIAG_MFMA_WORKGROUPS * 8 * iters * 16 * 32768 flop per launch: the ceiling of the matrix pipe with nothing else
 * running.  random_operands != 0 fills the operands with varied finite bit patterns (the sustained clock depends on
 * the data), 0 with constants.  sink: device, QG_DIAG_MFMA_WORKGROUPS * 512 floats (written so the loop is live).
 *
 * qg_diag_mfma_f64_loop: `workgroups` (1 .. 65536) workgroups of 256 threads; each wave issues iters rounds of 8
 * times 4 independent v_mfma_f64_4x4x4 on register operands: workgroups * 4 * iters * 8 * 2048 flop per launch, the
 * ceiling of the fp64 matrix pipe for the kernels of the subspace refresh.  sink: workgroups * 256 floats. */
#define QG_DIAG_MFMA_WORKGROUPS 512
int qg_diag_clock_probe(int64_t ticks_100mhz, int64_t* out2, void* stream);
int qg_diag_mfma_loop(int64_t iters, int random_operands, float* sink, void* stream);
int qg_diag_mfma_f64_loop(int64_t iters, int workgroups, float* sink, void* stream);

/* ---- Test helper: out[i] = u(seed, step, idx0 + i) for i < count, the uniform
 * draws of the stochastic-rounding generator, as fp32. */
int qg_sr_uniform(uint64_t seed, int64_t step, uint64_t idx0, int64_t count, float* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QGALORE_H */
