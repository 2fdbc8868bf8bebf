/*
 * elsaa.h -- C ABI of the ELSAA attention operator on AMD Instinct MI355X (gfx950).
 *
 * ELSAA ("Efficient Low-Rank and Sparse Approximation of Attention")
 * replaces dense softmax attention of one head by two branches and a fusion:
 *   - a sparse branch (sortLSH, Alg. 4; causal divide-and-conquer, Alg. 5):
 *     queries and keys are hashed with a sign hash, sorted by bucket, cut
 *     into equal blocks of b keys, and each query takes exact exp-weighted
 *     sums over its block: O_s = N_s / (d_s + eps), d_s = sum of e^{z};
 *   - a low-rank branch (RACE, Alg. 2; causal chunked form, Alg. 3): soft
 *     hypercube-hash features phi(x) of L tables with 2^gamma buckets give
 *     O_lr = Num / (Den + eps) and the denominator proxy d_lr = Den;
 *   - the denominator-aware fusion (Eq. m_sparse, Eq. elsaa_fusion_output,
 *     log-sum-exp form of Alg. 6):
 *        m = d_s / (d_s + lambda d_lr + eps),
 *        O = g_s * m * O_s + g_lr * O_lr.
 * The backward returns dQ, dK, dV (and optionally the gate gradients) with
 * the selection held fixed; the paper does not write a backward, it is the
 * exact gradient of the forward above.
 *
 * Tensor layout: Q, K, V, O, dO, dQ, dK, dV are [B, H, N, d_h] contiguous
 * row-major in the storage dtype (float32 or bfloat16); all accumulation is
 * float32.  Per-row outputs (lse, d_lr) are float32 [B, H, N].  The hash
 * projections are float32: W_sort [H, sort_bits, d_h] and
 * W_race [H, L, race_bits, d_h] with L = r / 2^race_bits, shared across the
 * batch.  gates is float32 [B, H, N, 2] = (g_sparse, g_lr) or NULL (all 1).
 *
 * Memory: every pointer except cfg is a device pointer owned by the caller.
 * The library never allocates or frees device memory and never synchronises
 * the caller's stream: it enqueues kernels and returns; results are valid
 * once the given stream has completed.  `saved` (elsaa_saved_bytes) is
 * written by elsaa_fwd and read by elsaa_bwd; `workspace`
 * (elsaa_workspace_bytes) is scratch for one call and may be reused by the
 * next call on the same stream.  Calls that share a workspace on different
 * streams race.
 *
 * Library-owned HIP objects: on its first call on a device, elsaa_fwd
 * creates one non-blocking stream of default priority and two events on
 * that device and keeps them until the process ends.  An elsaa_fwd call with
 * long lists to sort (where the overlap is worth the events) records an event
 * on the given stream, runs the sort of the selection on that second stream
 * while the given stream runs the low-rank branch, and makes the given stream
 * wait for the second stream before the sparse kernels (also when a launch in
 * between failed), so the call behaves as if everything ran on the given
 * stream; other calls use the given stream alone.  Concurrent elsaa_fwd calls on one
 * device share the second stream, so their sorts run one after another.
 *
 * Graph capture: elsaa_fwd and elsaa_bwd enqueue only kernels and event
 * record / wait pairs, so both can be captured into a HIP graph on the given
 * stream (the second stream joins the capture through the fork event) and
 * replayed; make one uncaptured call on the device first, which creates the
 * second stream and caches launch geometry.
 *
 * Errors: every entry point validates all arguments on the host before any
 * launch, so a rejected call writes nothing and leaves the stream untouched.
 * It returns a negative elsaa_status; elsaa_last_error() gives a message
 * (thread-local, valid until the next call on the same thread).
 */
#ifndef ELSAA_H
#define ELSAA_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ELSAA_OK = 0,
    ELSAA_ERR_INVALID_ARG = -1,   /* null pointer, out-of-range value */
    ELSAA_ERR_UNSUPPORTED = -2,   /* valid for the method, not implemented on the GPU path */
    ELSAA_ERR_WORKSPACE = -3,     /* saved / workspace buffer smaller than required */
    ELSAA_ERR_HIP = -4            /* a HIP launch or runtime call failed */
} elsaa_status;

typedef enum { ELSAA_F32 = 0, ELSAA_BF16 = 1, ELSAA_I8 = 2 } elsaa_dtype;   /* ELSAA_I8: outputs of elsaa_rms_norm_fwd only */

typedef struct {
    int32_t B, H, N, d_h;   /* batch, heads, sequence length, head dim (64 or 128);         */
                            /* GPU path: N <= 2^26 and N * d_h * element bytes < 2^32        */
    int32_t k;              /* sortLSH block size b: keys per sorted block, 1 <= k           */
    int32_t r;              /* RACE features L * 2^race_bits (the low-rank rank)             */
    int32_t race_bits;      /* gamma, hash bits per RACE table (GPU path: 4)                 */
    int32_t sort_bits;      /* gamma_sort, sign-hash bits of the sortLSH selector (1..8)      */
    int32_t n0;             /* causal base length N_0 of Alg. 5; <= 0 selects 2k             */
    int32_t causal;         /* 0: Alg. 1 / 2 / 4;  1: Alg. 6 / 3 / 5                          */
    int32_t dtype;          /* elsaa_dtype of Q,K,V,O,dO,dQ,dK,dV                             */
    float beta;             /* RACE temperature beta > 0 (Alg. 2)                            */
    float lambda;           /* fusion coefficient lambda >= 0 (Eq. m_sparse)                 */
    float eps;              /* numerical floor eps > 0                                       */
    float scale;            /* score scale tau; <= 0 selects 1/sqrt(d_h)                     */
    int32_t neighbors;      /* r >= 0: each sorted query block also sees the r neighbouring  */
                            /* sorted key blocks on each side (Sec. 6; 0 = the main setting)  */
    int32_t m_one;          /* 1: m_sparse = 1, the Sort_Lsh_RACE ablation (Sec. 7); 0: ELSAA */
} elsaa_config;

/* Number of causal recursion levels Lv (0 for non-causal).  Alg. 5 splits
 * every list longer than n0 into halves, padding an odd list with one zero
 * token first, so the lists at depth l all have L_l entries with L_0 = N,
 * L_{l+1} = ceil(L_l / 2), and Lv is the smallest depth with L_Lv <= n0.
 * Returns a negative status where a past half would have to hold a zero
 * token (fewer real tokens than half its list; never for n0 >= 2 * Lv). */
int elsaa_num_levels(const elsaa_config* cfg);

/* Entries of perm_q / perm_k per (b, h): N non-causal; causal the sum over
 * levels l < Lv of 2^l * L_{l+1} (= Lv * N / 2 when no list is padded). */
int64_t elsaa_perm_length(const elsaa_config* cfg);

/* Bytes of the `saved` buffer elsaa_fwd fills and elsaa_bwd reads, and of
 * the per-call scratch `workspace` (pass 0: elsaa_fwd / elsaa_select,
 * pass 1: elsaa_bwd).  Validates cfg. */
int elsaa_saved_bytes(const elsaa_config* cfg, size_t* bytes);
int elsaa_workspace_bytes(const elsaa_config* cfg, int pass, size_t* bytes);

/* Byte offsets inside `saved` (each 256-byte aligned):
 *   perm_q, perm_k  int32 sorted index lists (layout as elsaa_select);
 *   m               float32 [B,H,N] denominator-aware multiplier;
 *   o_sparse        float32 [B,H,N,d_h] sparse-branch output O_s (float32:
 *                   the backward's <dO, O_s> cancels against <dO, V_j> of
 *                   the dominant keys when attention is peaked);
 *   o_lowrank       storage dtype [B,H,N,d_h] low-rank output O_lr (its
 *                   weights are diffuse, so <dO, O_lr> has no such
 *                   cancellation);
 *   u_q, u_k        float32 [B,H,N,P] tanh of the RACE projections, t = tanh(W_race x),
 *                   of the Q and K rows (P = 4 L rounded up to 8, 16, 32 or 64;
 *                   padded tables 0);
 *   race_states     float32 RACE segment states phi(k) V' and phi(k) of the key
 *                   rows before each sequence segment (causal; the totals when
 *                   non-causal), [B*H][segments][r_p * d_h + r_p] with r_p = r
 *                   rounded up to 32, 64, 128 or 256; the segment length is an
 *                   internal choice, so only the library reads this region. */
typedef struct {
    size_t perm_q, perm_k, m, o_sparse, o_lowrank, u_q, u_k, race_states, total;
} elsaa_saved_layout;
int elsaa_get_saved_layout(const elsaa_config* cfg, elsaa_saved_layout* out);

/* Selection (Alg. 4 steps Hash / Sort / Partition; per level of Alg. 5).
 * Hash: bit t of a row x is set iff the float32 fused multiply-add chain
 * p = fma(W_sort[h][t][e], x[e], p) over e = 0..d_h-1 is > 0; the bucket key
 * is the position of that bit code in the reflected Gray sequence, so
 * neighbouring buckets differ in one bit ("sorted Hamming LSH", Sec. 3).
 * Sort: ascending by (key, token index), ties to the lower index.
 * Output (int32 token indices within one (b,h)):
 *   non-causal: perm_q, perm_k [B,H,N]; sorted block t = positions
 *               [t*k, (t+1)*k) and query block t sees key block t;
 *   causal:     perm_q, perm_k [B,H,P] (P = elsaa_perm_length); level l
 *               holds its 2^l segments in order, each giving its future
 *               half's queries (perm_q) and its past half's keys (perm_k)
 *               sorted, L_{l+1} entries each (elsaa_num_levels); a segment
 *               spans the real tokens [a, a + r) of its list, the rest of the
 *               list being Alg. 5's zero tokens, which trail future halves
 *               only: they take the bucket of the zero vector (key 0), sort
 *               after the real tokens of that bucket, and appear in perm_q
 *               as -1.  Without padding this is [B,H,Lv,N/2]. */
int elsaa_select(const elsaa_config* cfg, const void* Q, const void* K, const float* W_sort,
                 int32_t* perm_q, int32_t* perm_k, void* workspace, size_t workspace_bytes,
                 hipStream_t stream);

/* The selection above for callers that cannot allocate: code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation.  Same
 * arguments and results as elsaa_select (perm_q, perm_k are the caller's),
 * without `workspace`: the hash keys (2 * B*H*N bytes, each half 256-byte
 * aligned) go to a fixed 32 MiB device array inside the library, which every
 * device the library runs on holds until the process ends.  Rejects
 * B*H*N above 16777088 tokens with ELSAA_ERR_WORKSPACE before any launch.
 * Calls no allocating routine (the device address of the array is looked up
 * once per device, on the first call with that device current).  All calls
 * on one device share the array: calls that overlap on one device (other
 * streams, other threads) race; calls on one stream are ordered. */
int elsaa_select_noalloc(const elsaa_config* cfg, const void* Q, const void* K, const float* W_sort,
                         int32_t* perm_q, int32_t* perm_k, hipStream_t stream);

/* Forward (Alg. 1 / Alg. 6 without the projections).  gates is [B,H,N,2]
 * float32 (g_sparse, g_lr) or NULL (all 1); lambda_rows is the per-token
 * coefficient lambda_i of Eq. m_sparse, [B,H,N] float32 >= 0, or NULL (the
 * scalar cfg->lambda for every token).  Writes
 *   O        [B,H,N,d_h] storage dtype, fused output;
 *   lse      [B,H,N] float32, log d_sparse (log of the sparse denominator);
 *   d_lr     [B,H,N] float32, RACE denominator proxy Den;
 *   saved    selection, m, O_s, O_lr, the RACE projections and states for
 *            the backward (elsaa_saved_layout). */
int elsaa_fwd(const elsaa_config* cfg, const void* Q, const void* K, const void* V,
              const float* W_sort, const float* W_race, const float* gates, const float* lambda_rows,
              void* O, float* lse, float* d_lr, void* saved, size_t saved_bytes,
              void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Backward.  dO is the upstream gradient of O; gates, lambda_rows, lse, d_lr
 * and saved are what elsaa_fwd was given / wrote for the same inputs.
 * Writes dQ, dK, dV [B,H,N,d_h] (storage dtype) and, when not NULL,
 * dgates [B,H,N,2] float32 (d/dg_sparse, d/dg_lr) and dlambda [B,H,N]
 * float32 (d/dlambda_i; the gradient of a scalar lambda is their sum, that
 * of lambda = exp(l) is lambda times it; zero when m_one).  W_sort is not
 * read (the selection comes from saved) and may be NULL. */
int elsaa_bwd(const elsaa_config* cfg, const void* Q, const void* K, const void* V,
              const float* W_sort, const float* W_race, const float* gates, const float* lambda_rows,
              const void* dO, const float* lse, const float* d_lr, const void* saved, size_t saved_bytes,
              void* dQ, void* dK, void* dV, float* dgates, float* dlambda,
              void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Token-wise rules that feed the fusion: the gate network and the
 * query-dependent lambda.
 *   gates (Sec. 3.3, Alg. 1; the two-layer SiLU MLP with two independent,
 *   unnormalised sigmoid outputs of the experimental setup):
 *       (g_sparse, g_lr)_i = sigmoid(W2 SiLU(W1 q_i + b1) + b2)
 *   lambda (the query-dependent coefficient of the ELSAA configuration
 *   appendix, q_i detached from this path):
 *       lambda_i = max(lambda_min, c + sigmoid(w . q_i + b))
 * q_i is row i of the head's Q; every head has its own parameters.  The
 * caller keeps c >= 0 (it is used as given); lambda_min is 1e-6 in the paper.
 * Layouts (float32, contiguous, W1 and w 16-byte aligned):
 *   W1 [H, G, d_h], b1 [H, G], W2 [H, 2, G] (row 0 -> g_sparse), b2 [H, 2];
 *   w [H, d_h], b [H], c [H].
 * gate_hidden G is 0 (no gate network), 64 or 128 (the paper's text and
 * vision widths); lambda_rule is 0 or 1; at least one must be on.  Pointers
 * of a rule that is off are not read. */
typedef struct {
    int32_t gate_hidden;
    const float* W1;
    const float* b1;
    const float* W2;
    const float* b2;
    int32_t lambda_rule;
    const float* lam_w;
    const float* lam_b;
    const float* lam_c;
    float lambda_min;
} elsaa_token_rules;

/* Forward of the rules: writes gates [B,H,N,2] (when gate_hidden > 0) and
 * lambda_rows [B,H,N] (when lambda_rule), both float32, ready to pass to
 * elsaa_fwd / elsaa_bwd.  Q is the operator's Q (cfg->dtype storage). */
int elsaa_token_rules_fwd(const elsaa_config* cfg, const elsaa_token_rules* rules, const void* Q,
                          float* gates, float* lambda_rows, hipStream_t stream);

/* Bytes of the workspace elsaa_token_rules_bwd needs (per-workgroup partial
 * sums of the parameter gradients). */
int elsaa_token_rules_workspace_bytes(const elsaa_config* cfg, const elsaa_token_rules* rules,
                                      size_t* bytes);

/* Backward of the rules, given dgates and dlambda (what elsaa_bwd wrote):
 *   dQ      accumulated IN PLACE: dQ += d/dQ of sum(dgates * gates), the
 *           gate network's contribution (the lambda path is detached);
 *           NULL skips it;
 *   dW1, db1, dW2, db2, dlam_w, dlam_b, dlam_c: parameter gradients with the
 *           shapes of the parameters, summed over B and N (overwritten);
 *           any may be NULL.
 * dgates is read when gate_hidden > 0, dlambda when lambda_rule.  The sums
 * are taken in a fixed order (deterministic). */
int elsaa_token_rules_bwd(const elsaa_config* cfg, const elsaa_token_rules* rules, const void* Q,
                          const float* dgates, const float* dlambda, void* dQ,
                          float* dW1, float* db1, float* dW2, float* db2,
                          float* dlam_w, float* dlam_b, float* dlam_c,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Dense projections of the attention block (Alg. 1 and Alg. 6: Q = X W_Q,
 * K = X W_K, V = X W_V before the operator, O_head W_O after it; the paper
 * keeps these matrices dense, Sec. 1 and the parameter-overhead appendix).
 *
 * elsaa_gemm computes C = op(A) op(B) with op(A) [M,K], op(B) [K,N],
 * C [M,N], bfloat16 operands and float32 accumulation; C is bfloat16 or
 * float32 (c_dtype).  op(X) = X, or X^T when trans_x = 1, of the STORED
 * matrix X: A is stored [M,K] (trans_a = 0) or [K,M] (trans_a = 1), B is
 * stored [K,N] (trans_b = 0) or [N,K] (trans_b = 1).
 *
 * Each stored matrix (and C) is in one of two layouts, chosen per operand:
 *   plain       row-major with row stride ld (elements), ld >= its columns;
 *   head-major  (x_heads = Hx > 0) the stored matrix of R rows and Hx * dh
 *               columns is kept as [R / seq][Hx][seq][dh] contiguous: row
 *               r = b * seq + n, column c = h * dh + e lives at
 *               ((b * Hx + h) * seq + n) * dh + e.  This is the [B,H,N,d_h]
 *               layout of Q, K, V, O and their gradients, so the projections
 *               read and write attention tensors without a reshape copy.
 *               dh = columns / Hx must be a multiple of 8 and R a multiple
 *               of seq; ld is ignored.
 * Requirements: M, N, K >= 1 and multiples of 8, plain ld multiples of 8,
 * pointers 16-byte aligned, A / B / C not overlapping.  A and B are never
 * written.  When the output has few tiles and K is long, the K range is
 * split over workgroups whose float32 partial products go to `workspace`
 * (elsaa_gemm_workspace_bytes; 0 when no split is used) and are summed in a
 * fixed order, so results are deterministic run to run. */
typedef struct {
    int32_t M, N, K;
    int32_t trans_a, trans_b;
    int64_t lda, ldb, ldc;
    int32_t a_heads, b_heads, c_heads;   /* 0 = plain, Hx > 0 = head-major */
    int32_t seq;                         /* rows per sequence of head-major operands */
    int32_t c_dtype;                     /* elsaa_dtype of C */
} elsaa_gemm_desc;

int elsaa_gemm_workspace_bytes(const elsaa_gemm_desc* desc, size_t* bytes);
int elsaa_gemm(const elsaa_gemm_desc* desc, const void* A, const void* B, void* C,
               void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Root-mean-square norm of the residual stream in front of a block:
 *     s = x + residual,   y_j = s_j rho w_j,   rho = (mean_j s_j^2 + eps)^(-1/2)
 * for each of `rows` rows of `cols` values.  Rows are `ld` elements apart
 * (ld >= cols); the weight is float32 [cols].  Sums and the norm are float32
 * whatever the storage type, and y is formed from the unrounded s.
 * (Squares are summed as they are: where a row's sum of them passes 3.4e38, rho and
 * the finite y are 0, and the row has no meaningful gradient.)
 *
 * elsaa_rms_norm_fwd writes s to `sum` in the storage type (NULL: not kept;
 * without a residual s is x) and y as y_dtype says:
 *   dtype      y in the storage type, `scale` unused;
 *   ELSAA_I8   8-bit values with one float32 scale a row, y_j ~ scale * q_j:
 *              scale = max_j |y_j| / 127, q_j = y_j / scale rounded to
 *              nearest, ties to even.  A row of zeros has scale 0; a row with
 *              an infinity or NaN has scale NaN and q 0.
 * `sum` may be x or the residual itself, y (storage type) may be x or the residual,
 * each at the same row stride: a row is read before it is written.  Another stride, and
 * sum and y at one address, are refused; buffers must not overlap otherwise.
 *
 * elsaa_rms_norm_bwd is the gradient at the stored s (argument X, ldx), from
 * dY (ldy) and, when not NULL, the residual stream's own gradient dS (ldr):
 *     dx_j = rho (w_j dy_j - s_j rho^2 mean_i(w_i dy_i s_i)) + ds_j   (dX, lds)
 *     dw_j = sum over rows of dy_j s_j rho                         (float32)
 * dX is the gradient of x and of the residual alike; it may be dS, dY or X
 * itself at the same stride (another is refused).  dweight may be NULL.  dw is summed over the workgroups'
 * partial sums in `workspace` (elsaa_rms_norm_workspace_bytes; 0 without dweight need
 * not be passed) in a fixed order, so it is the same from run to run.
 * Requirements: rows >= 1, 1 <= cols <= 16384, pointers aligned to their
 * element.  Rows of any alignment work; 16-byte aligned buffers whose cols and strides
 * are multiples of 8 are read and written 16 bytes at a time. */
typedef struct {
    int64_t rows;
    int32_t cols;
    int32_t dtype;                  /* storage: ELSAA_F32 or ELSAA_BF16 */
    int32_t y_dtype;                /* forward: dtype or ELSAA_I8 */
    float eps;                      /* > 0 */
    int64_t ldx, ldr, lds, ldy;     /* row strides in elements */
} elsaa_norm_desc;

int elsaa_rms_norm_fwd(const elsaa_norm_desc* desc, const void* X, const void* residual, const float* weight,
                       void* sum, void* Y, float* scale, hipStream_t stream);
int elsaa_rms_norm_workspace_bytes(const elsaa_norm_desc* desc, size_t* bytes);
int elsaa_rms_norm_bwd(const elsaa_norm_desc* desc, const void* X, const float* weight, const void* dY,
                       const void* dS, void* dX, float* dweight, void* workspace, size_t workspace_bytes,
                       hipStream_t stream);

/* 8-bit rows with one scale a row, as elsaa_rms_norm_fwd's 8-bit output:
 * scale_i = max_j |x_ij| / 127, q_ij = x_ij / scale_i to nearest, ties to even.
 * X is a rows x cols matrix, plain (row stride ld) or head-major (heads > 0:
 * [rows / seq][heads][seq][cols / heads] contiguous, cols / heads a power of
 * two >= 8, as elsaa_gemm's operands); Q is plain with row stride ldq.  Weights (a row for each output
 * channel) are laid out once, attention outputs on every call.
 * 1 <= cols <= 16384. */
typedef struct {
    int64_t rows;
    int32_t cols;
    int32_t dtype;                  /* of X: ELSAA_F32 or ELSAA_BF16 */
    int64_t ld, ldq;
    int32_t heads, seq;             /* head-major X; heads = 0: plain */
} elsaa_quant_desc;

int elsaa_quantize_rows(const elsaa_quant_desc* desc, const void* X, int8_t* Q, float* scale, hipStream_t stream);

/* Product of 8-bit rows and 8-bit weights with a scale for each row (token)
 * and each output channel:
 *     C_ij = a_scale_i b_scale_j sum_k A_ik B_jk
 * A [M, K] (row stride lda), B [N, K] (row stride ldb: a row for each channel, the
 * transpose of elsaa_gemm's B), 8-bit two's complement; the sums are exact
 * 32-bit integers, scaled in float32 (by a_scale, then b_scale: infinite where the sum times
 * a_scale passes 3.4e38) and rounded once to c_dtype.  C is plain (ldc) or
 * head-major (c_heads > 0, seq) as in elsaa_gemm, with any power of two >= 8 as head
 * width.  Requirements: 1 <= M, N <= 2^30, 1 <= K <= 131071 (the largest whose sums fit 32 bits), fewer
 * than 2^24 tiles of C (256 x 256 where K is a multiple of 16 and at least 128, else 128 x 128), lda, ldb
 * multiples of 16 (bytes), A and B 16-byte aligned, C aligned to its element; K need not be a multiple of
 * anything (bytes between K and the next multiple of 16 are read and ignored).
 * Long sums with few output tiles are split over workgroups whose integer
 * partial sums go to `workspace` (elsaa_gemm_i8_workspace_bytes; 0 when none is used). */
typedef struct {
    int32_t M, N, K;
    int64_t lda, ldb, ldc;
    int32_t c_heads, seq;
    int32_t c_dtype;                /* ELSAA_F32 or ELSAA_BF16 */
} elsaa_gemm_i8_desc;

int elsaa_gemm_i8_workspace_bytes(const elsaa_gemm_i8_desc* desc, size_t* bytes);
int elsaa_gemm_i8(const elsaa_gemm_i8_desc* desc, const int8_t* A, const float* a_scale, const int8_t* B,
                  const float* b_scale, void* C, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Linear attention with a decay for each head, the attention of blocks that
 * are served token by token: with lambda_h = exp(log_decay[h]),
 *     S_t = lambda_h S_{t-1} + k_t v_t^T      (d_h x d_h, float32)
 *     o_t = tau q_t^T S_t                     (tau = scale; <= 0: 1/sqrt(d_h))
 * log_decay is float32 [H], each <= 0 (0: no decay; -infinity: a token sees
 * itself only); it is a constant of the head and has no gradient.
 *
 * Q, K, V, O and their gradients are [B, H, N, d_h] in the storage type, the
 * inner three dimensions contiguous and batches `*_batch` elements apart (0:
 * H N d_h), so they can be head ranges of one projection buffer
 * [B, 3H, N, d_h] as AttentionBlock keeps it.  States are float32
 * [B, H, d_h, d_h] contiguous, row index k, column index v.
 *
 * lengths: int32 [B] on the device or NULL (every sequence has N tokens);
 * values are clamped to 0 .. N.  Tokens at and behind a sequence's length are not
 * read; their rows of O are left as they were, or set to zero where zero_tail is
 * not 0, their rows of dQ, dK, dV are set to zero.
 *
 * elsaa_decay_fwd: state is S_0 (NULL: zero); state_out, when not NULL, receives S behind the last
 * token (it may be `state` itself).
 * elsaa_decay_bwd: dstate_out is the gradient of state_out (NULL: zero), and dstate, when
 * not NULL, receives that of `state` (it may be dstate_out itself).
 * elsaa_decay_step: one token for each sequence (N = 1 in the descriptor),
 * state -> state_out (may be the same buffer).
 * No output may overlap an input or another output, the states above excepted (the
 * same address is refused).
 * The chunked form splits a sequence over workgroups, whose states go to
 * `workspace` (elsaa_decay_workspace_bytes, pass 0: fwd, 1: bwd).  All sums have a
 * fixed order.  An infinity or NaN of a token reaches what the recurrence says: outputs and dQ of
 * that and later tokens (a query only its own output), dK and dV of that and earlier ones.
 * (The segment that holds one is read out token by token, 1.2 to 1.8 us each.)
 * Limits: d_h 64 or 128; N * d_h * element bytes < 2^32; B * H <= 2^22. */
typedef struct {
    int32_t B, H, N, d_h;
    int32_t dtype;                  /* ELSAA_F32 or ELSAA_BF16 */
    float scale;
    int64_t q_batch, k_batch, v_batch, o_batch;         /* o_batch: O and dO */
    int64_t dq_batch, dk_batch, dv_batch;
    int32_t zero_tail;                                  /* forward with lengths: rows of O behind them become zero */
} elsaa_decay_desc;

int elsaa_decay_workspace_bytes(const elsaa_decay_desc* desc, int pass, size_t* bytes);
int elsaa_decay_fwd(const elsaa_decay_desc* desc, const void* Q, const void* K, const void* V, const float* log_decay,
                    const float* state, const int32_t* lengths, void* O, float* state_out,
                    void* workspace, size_t workspace_bytes, hipStream_t stream);
int elsaa_decay_bwd(const elsaa_decay_desc* desc, const void* Q, const void* K, const void* V, const float* log_decay,
                    const void* dO, const float* state, const float* dstate_out, const int32_t* lengths,
                    void* dQ, void* dK, void* dV, float* dstate, void* workspace, size_t workspace_bytes,
                    hipStream_t stream);
int elsaa_decay_step(const elsaa_decay_desc* desc, const void* Q, const void* K, const void* V,
                     const float* log_decay, const float* state, void* O, float* state_out, hipStream_t stream);

/* Opt-in kernel timing.  While enabled, every kernel launch of the library
 * is bracketed by two HIP events recorded on its stream (one extra event pair
 * per launch, no synchronisation); elsaa_profile_count / elsaa_profile_get
 * wait for the recorded launches and report, per kernel name, the summed
 * event time in milliseconds and the number of launches.  Enabling clears
 * the previous totals.  Process-wide; disabled by default. */
int elsaa_profile_enable(int on);
int elsaa_profile_count(void);
int elsaa_profile_get(int index, char* name, size_t name_len, double* total_ms, int64_t* launches);

const char* elsaa_status_string(int status);
const char* elsaa_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ELSAA_H */
