/*
 * tlq.h - C ABI of libtlq: the data-parallel hot path of TLQ's layer-wise
 * scale search on one AMD MI355X (gfx950).
 *
 * What the library computes (paper: "Rethinking Practical and Efficient
 * Quantization Calibration for Vision-Language Models"):
 *   for one linear layer with weights W [c_out, c_in] and calibration tokens
 *   X [n_tok, c_in], and for every candidate exponent alpha_k of a grid,
 *     s_k      = x_stat ^ alpha_k                        (Sec. 3.1.2, scale eq.)
 *     Wq_k     = Q_w(W * diag(s_k))                       (Sec. 3.2.1, f_q)
 *     Yq_k     = (X * diag(s_k)^-1) * Wq_k^T              (Sec. 2.2, smoothing eq.)
 *     L_k      = sum_t w_t * (1/c_out) * sum_o (Y_ref[t,o] - Yq_k[t,o])^2
 *                                                         (Sec. 3.2.1, objective)
 *   and returns k* = argmin_k L_k together with s_{k*}.  Q_w is round-to-
 *   nearest integer quantisation (Sec. 2.2) on a min/max grid per group of
 *   consecutive input channels; activations stay in 16-bit floating point.
 *
 * Conventions that hold for every entry point
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The
 *     library never allocates, frees or keeps device memory; scratch comes
 *     from the caller's `workspace` (size from the matching *_workspace_bytes
 *     query; 256-byte aligned).  A workspace that is too small gives
 *     TLQ_ERR_WORKSPACE and nothing is launched.
 *   - `stream` is the caller's hipStream_t passed as void* (NULL = the null
 *     stream).  All work is enqueued on it in order; no entry point
 *     synchronises with the host or copies to the host.  Outputs are device
 *     resident and valid once the stream reaches the end of the call.
 *   - The return value reports argument validation and launch errors only.
 *     Validation (every status except TLQ_ERR_LAUNCH) happens before any HIP call:
 *     nothing was launched and nothing was written.  TLQ_ERR_LAUNCH means the HIP
 *     runtime refused a launch part-way through the call: kernels enqueued before it
 *     may still run and the outputs and the workspace must be treated as undefined.
 *     Faults inside a kernel surface at the caller's next synchronisation.
 *   - Matrices are row-major with a row stride (`ld*`) in ELEMENTS.  16-bit
 *     matrices need 16-byte aligned base pointers and strides that are
 *     multiples of 8; otherwise TLQ_ERR_ALIGN.  c_in must be a multiple of 8
 *     and of `group` (TLQ_ERR_SHAPE otherwise).
 *   - Calls on different streams may run concurrently if their workspaces and
 *     outputs are disjoint.  The library keeps no state between calls except (a) the
 *     optional per-kernel timing (tlq_profile_*: one process-wide table behind a mutex)
 *     and (b) the fixed scratch array of tlq_x_stat_static.
 *   - Float vectors that are read 16 bytes at a time (`s` of tlq_fake_quant and
 *     tlq_apply_best) must be 16-byte aligned; `group` must be 0 or a multiple of 8
 *     (TLQ_ERR_UNSUPPORTED otherwise); uint8 code matrices must be 8-byte aligned.
 *   - act_bits > 0 (Sec. 3.2.1 f_q with Q_a; quantiser of Sec. 2.2 per token row):
 *     xt = x * float(1/s); sigma_t = max(max_c |xt|, 1e-5) / (2^(n-1)-1);
 *     code = clip(rint(xt/sigma_t), -2^(n-1), 2^(n-1)-1); f_q = sigma_t * code . deq^T.
 *     float arithmetic, round half to even.  Applies to tlq_scale_search,
 *     tlq_weighted_layer_err and tlq_apply_best.
 *   - x_dtype = BF16: inputs and 16-bit outputs are bf16.  Operands the library
 *     computes itself (the folded weights deq/s) are kept in fp16, and the tokens
 *     are re-expressed in fp16 in the workspace (exact for bf16 values after a
 *     power-of-two prescale), so bf16 inputs get the same loss accuracy as fp16.
 */
#ifndef TLQ_H
#define TLQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TLQ_VERSION 100 /* 0.1.0 */
#define TLQ_MAX_ALPHA 64 /* largest alpha grid one call accepts */

typedef enum {
  TLQ_OK = 0,
  TLQ_ERR_NULL = 1,        /* a required pointer is NULL */
  TLQ_ERR_SHAPE = 2,       /* a size is non-positive or inconsistent */
  TLQ_ERR_UNSUPPORTED = 3, /* a parameter value this build does not implement */
  TLQ_ERR_WORKSPACE = 4,   /* workspace missing or smaller than the query says */
  TLQ_ERR_ALIGN = 5,       /* pointer or stride alignment */
  TLQ_ERR_LAUNCH = 6       /* the HIP runtime rejected a launch */
} tlq_status;

typedef enum { TLQ_F16 = 0, TLQ_BF16 = 1, TLQ_F32 = 2 } tlq_dtype;

/* Plain-old-data parameter block, passed by const pointer. */
typedef struct tlq_params {
  uint32_t struct_size; /* = sizeof(tlq_params); anything else: TLQ_ERR_UNSUPPORTED */
  int32_t bits;         /* weight bits, 2..8 */
  int32_t group;        /* input channels per quantisation group; 0 = whole row */
  int32_t symmetric;    /* 0 = asymmetric min/max grid, 1 = symmetric max|.| grid */
  int32_t act_bits;     /* 0 = activations not quantised; 2..8 = per-token symmetric Q_a */
  int32_t xstat_kind;   /* 0 = mean |x| over tokens, 1 = max |x| over tokens */
  int32_t x_dtype;      /* tlq_dtype of X and of W and of the MFMA operands: F16 or BF16 */
  int32_t yref_dtype;   /* tlq_dtype of Y_ref (and of tlq_ref_output's result) */
} tlq_params;

const char* tlq_status_string(int status);
int tlq_version(void);

/* ---- S0: per-channel activation statistic (Sec. 3.1.2, x_stat; mean form of
 * the ablation table, or max).  x_stat[c] = (1/n_tok) sum_t |X[t,c]| rounded
 * once to float (sum and division in double), or max_t |X[t,c]|.
 * x_stat: out, float [c_in]. */
size_t tlq_x_stat_workspace_bytes(int64_t n_tok, int64_t c_in);
tlq_status tlq_x_stat(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                      const tlq_params* p, float* x_stat,
                      void* workspace, size_t workspace_bytes, void* stream);

/* ---- tlq_x_stat for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same kernels, same
 * result bit for bit as tlq_x_stat, but the partial sums live in a fixed 16 MiB device
 * array inside the library (one copy per GPU, held until the process ends) instead of a
 * caller workspace.  The call allocates and frees nothing, on the device or through any
 * library.  Limits: c_in <= TLQ_X_STAT_STATIC_MAX_C_IN (TLQ_ERR_WORKSPACE beyond it);
 * per-kernel timing must be off (TLQ_ERR_UNSUPPORTED while tlq_profile_enable(1) is in
 * force, because timing creates HIP events).  The stream must belong to the device that is
 * current at the call.  All calls on one GPU share that GPU's array: calls that overlap in
 * time on one GPU (different streams or threads) race on it and give wrong results;
 * serialise them.  Nothing in the array needs to survive between calls. */
#define TLQ_X_STAT_STATIC_MAX_C_IN 16384
tlq_status tlq_x_stat_static(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                             const tlq_params* p, float* x_stat, void* stream);

/* ---- gradient-guided token selection (Sec. 3.1.2).  G holds per-sample gradients with
 * respect to the layer input, sample major: [n_samples * n_pos, c] x_dtype.
 *   tlq_token_importance: sum_n[n] = sum_b ||g_{b,n}||, n < n_pos (gradient-statistic eq.);
 *     the norm is mean_c |g| (l2 = 0, the text's description) or the Euclidean norm (l2 = 1);
 *     double accumulation in a fixed order; sum_n: out double [n_pos].
 *   tlq_topk_mask: I = Top_k({sum_n}) (selection eq.; the paper keeps k = n_pos/2); ties go
 *     to the lower position; mask: out uint8 [n_pos], 1 = selected.  n_pos <= 65536.
 *   tlq_x_stat_masked: x_stat[c] = max over rows t with pos_mask[t mod period] != 0 of
 *     |X[t,c]| (x_stat eq.; X stacks samples of `period` positions); workspace as tlq_x_stat.
 * The result feeds tlq_scale_search through x_stat_in. */
size_t tlq_token_importance_workspace_bytes(int64_t n_samples, int64_t n_pos);
tlq_status tlq_token_importance(const void* G, int64_t n_samples, int64_t n_pos, int64_t c,
                                int64_t ldg, int32_t l2, const tlq_params* p, double* sum_n,
                                void* workspace, size_t workspace_bytes, void* stream);
tlq_status tlq_topk_mask(const double* sum_n, int64_t n_pos, int64_t k, uint8_t* mask, void* stream);
tlq_status tlq_x_stat_masked(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                             const uint8_t* pos_mask, int64_t period, const tlq_params* p,
                             float* x_stat, void* workspace, size_t workspace_bytes, void* stream);

/* ---- S1: candidate scales (Sec. 3.1.2 scale eq.; Sec. 3.2.1 per-layer form).
 * s_table[k,c] = float( pow( double(max(x_stat[c], 2^-14)), double(alpha[k]) ) ).
 * x_stat: in, float [c_in]; alpha_grid: in, float [n_alpha];
 * s_table: out, float [n_alpha, c_in]. */
tlq_status tlq_scale_table(const float* x_stat, int64_t c_in, const float* alpha_grid,
                           int32_t n_alpha, float* s_table, void* stream);

/* ---- S2: fake quantisation of W * diag(s) (Sec. 2.2 quantiser in min/max
 * form; Sec. 3.2.1 Q_w(W * scale)).  All grid arithmetic is float, one
 * rounding per operation, round-half-to-even:
 *   ws = W*s; rng = max(max_g ws - min_g ws, 1e-5); delta = rng/(2^bits-1);
 *   zp = clip(rint(-min/delta), 0, 2^bits-1);
 *   q  = clip(rint(ws/delta) + zp, 0, 2^bits-1);  deq = (q - zp)*delta.
 * (symmetric=1: delta = max(max_g|ws|,1e-5)/(2^(bits-1)-1), q = clip(rint(ws/
 * delta), -2^(bits-1), 2^(bits-1)-1), stored codes are q + 2^(bits-1), zp =
 * 2^(bits-1).)
 * W: in [c_out, c_in] x_dtype; s: in float [c_in] or NULL (= ones).
 * Outputs, each may be NULL (skipped): codes uint8 [c_out, c_in] (dense),
 * zp uint8 [c_out, G], delta float [c_out, G], G = c_in/group;
 * Wdq [c_out, c_in] x_dtype with row stride ld_dq = deq rounded to x_dtype. */
tlq_status tlq_fake_quant(const void* W, int64_t c_out, int64_t c_in, int64_t ldw,
                          const float* s, const tlq_params* p,
                          uint8_t* codes, uint8_t* zp, float* delta,
                          void* Wdq, int64_t ld_dq, void* stream);

/* ---- Q_a alone (Sec. 3.2.1 Q_a(x/scale); quantiser of Sec. 2.2 per token row; formula in
 * the conventions above).  Needs act_bits > 0.  inv_s: float [c_in] or NULL (ones).
 * codes: out [n_tok, c_in] dense, the integer codes stored as fp16 numbers (exact);
 * sigma: out float [n_tok]. */
tlq_status tlq_act_fake_quant(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                              const float* inv_s, const tlq_params* p, void* codes, float* sigma,
                              void* stream);

/* ---- S3+S4 for one given dequantised weight matrix (Sec. 3.2.1 objective
 * with f_q = (X*inv_s) Wdq^T):
 *   err[t] = (1/c_out) sum_o (Y_ref[t,o] - sum_c X[t,c]*inv_s[c]*Wdq[o,c])^2
 *   loss   = sum_t token_w[t] * err[t]
 * X [n_tok,c_in], Wdq [c_out,c_in]: x_dtype; inv_s: float [c_in] or NULL (ones);
 * Y_ref [n_tok,c_out] yref_dtype; token_w float [n_tok] (used as given).
 * loss: out float [1]; per_token_err: out float [n_tok] or NULL.
 * The operand that enters the matrix cores is round16(Wdq * inv_s); on problems with only a
 * handful of outputs that rounding can show in the loss beyond 1e-3 (tlq_scale_search, which
 * also sees W, avoids it there).
 * Where the outputs are few tiles the query asks for the room of tiles of 128 rows; a
 * workspace with room for those of 256 rows (4 bytes for each of them and for n_tok of every 256
 * outputs instead of every 128) is taken too, and the call is slower. */
size_t tlq_weighted_layer_err_workspace_bytes(int64_t n_tok, int64_t c_in, int64_t c_out,
                                              const tlq_params* p);
tlq_status tlq_weighted_layer_err(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                                  const void* Wdq, int64_t c_out, int64_t ldw,
                                  const float* inv_s,
                                  const void* Y_ref, int64_t ldy, const float* token_w,
                                  const tlq_params* p, float* loss, float* per_token_err,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* ---- S0..S5: the search (Sec. 3.2.1: r* = argmin_r E||f_fp(x) - f_q(x; x_stat^r)||^2).
 * x_stat_in: float [c_in] or NULL (then computed from X per xstat_kind).
 * alpha_grid: float [n_alpha], 1 <= n_alpha <= TLQ_MAX_ALPHA.
 * Outputs: best_scales float [c_in] (= s_table[best_idx]); best_idx int32 [1]
 * (first minimum; -1 if no candidate has a finite loss); losses float
 * [n_alpha] (+inf where not finite); s_table_out float [n_alpha, c_in] or NULL.
 * Arithmetic: 16-bit matrix-core operands, float accumulation.  Without
 * activation quantisation the operand is the folded weight
 * round16(deq_k / s_k); from 6 weight bits on, and for problems smaller than
 * 256 x 256 outputs, it is the difference round16(deq_k / s_k - W) and the
 * residual is formed against Y_ref - X W^T kept in float (one more
 * contraction and n_tok x c_out floats of workspace), because there the
 * rounding of the folded weight itself would show in the loss. */
size_t tlq_scale_search_workspace_bytes(int64_t n_tok, int64_t c_in, int64_t c_out,
                                        int32_t n_alpha, const tlq_params* p);
tlq_status tlq_scale_search(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                            const void* W, int64_t c_out, int64_t ldw,
                            const void* Y_ref, int64_t ldy, const float* token_w,
                            const float* alpha_grid, int32_t n_alpha, const tlq_params* p,
                            const float* x_stat_in,
                            float* best_scales, int32_t* best_idx, float* losses,
                            float* s_table_out,
                            void* workspace, size_t workspace_bytes, void* stream);

/* ---- tokens prepared once for several calls on the same X (Sec. 3.2.1: q/k/v and gate/up
 * are searched, and then propagated, on one exposed input).  With x_dtype = BF16 and act_bits = 0
 * every search and every propagation first re-expresses X in fp16 (see the conventions above);
 * tlq_prepare_tokens does that once into a caller buffer of tlq_prepared_tokens_bytes bytes
 * (256-byte aligned; 0 = these parameters need no preparation and `prepared` may be NULL), and
 * the *_prepared variants below take that buffer instead of repeating the conversion.  They
 * are otherwise identical to tlq_scale_search / tlq_apply_best (same arguments, same results
 * bit for bit); prepared = NULL makes them the plain calls.  The buffer must have been
 * filled from the same X, n_tok, c_in and parameters on the same stream order. */
size_t tlq_prepared_tokens_bytes(int64_t n_tok, int64_t c_in, const tlq_params* p);
tlq_status tlq_prepare_tokens(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                              const tlq_params* p, void* prepared, size_t prepared_bytes,
                              void* stream);
tlq_status tlq_scale_search_prepared(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                                     const void* W, int64_t c_out, int64_t ldw,
                                     const void* Y_ref, int64_t ldy, const float* token_w,
                                     const float* alpha_grid, int32_t n_alpha, const tlq_params* p,
                                     const float* x_stat_in,
                                     float* best_scales, int32_t* best_idx, float* losses,
                                     float* s_table_out,
                                     void* workspace, size_t workspace_bytes, void* stream,
                                     const void* prepared);
tlq_status tlq_apply_best_prepared(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                                   const void* W, int64_t c_out, int64_t ldw, const float* s,
                                   const tlq_params* p, void* X_next, int64_t ld_next,
                                   void* workspace, size_t workspace_bytes, void* stream,
                                   const void* prepared);

/* ---- the weight-only search in second-moment form (Sec. 3.2.1 objective with f_q linear in x,
 * i.e. act_bits == 0).  For f_fp(x) = x W^T and f_q(x) = x What_k^T the objective
 *   sum_t token_w[t] (1/c_out) ||f_fp(x_t) - f_q(x_t)||^2  =  (1/c_out) sum_o d_o^T G d_o,
 *   d_o = row o of W - What_k,   G = sum_t token_w[t] x_t x_t^T   [c_in, c_in],
 * so the tokens enter through G alone.  G does not depend on the candidate or on the linear:
 * linears that share an input (q/k/v, gate/up) share one G, and a candidate then costs
 * 2 c_out c_in^2 flops instead of 2 n_tok c_in c_out.  It pays when n_tok is well above c_in.
 * The target is the exact product x W^T (no rounded Y_ref enters), and no per-token error exists.
 *
 * tlq_token_gram writes a device-resident representation of G into `gram`
 * (tlq_token_gram_bytes(c_in) bytes, 256-byte aligned, caller-owned): a double `factor` at byte 0,
 * float col_scale[c_in] at byte 256, then (256-byte aligned) fp16 C[c_in, c_in], with
 *   G[i,j] = factor * col_scale[i] * col_scale[j] * C[i,j];
 * col_scale holds powers of two chosen so that |C| <= 2 whatever the spread of the channel
 * magnitudes.  Tokens must lie inside the fp16 range (|x| < 65504) - beyond it the losses come out
 * non-finite.  Workspace from the query.
 * tlq_scale_search_gram is tlq_scale_search with (X, Y_ref, token_w) replaced by `gram`; x_stat
 * [c_in] is required (tlq_x_stat of the same X).  act_bits != 0 -> TLQ_ERR_UNSUPPORTED.  Outputs,
 * non-finite rule and tie rule as for tlq_scale_search. */
size_t     tlq_token_gram_bytes(int64_t c_in);
size_t     tlq_token_gram_workspace_bytes(int64_t n_tok, int64_t c_in);
tlq_status tlq_token_gram(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                          const float* token_w /*[n_tok]*/, const tlq_params* p,
                          void* gram, size_t gram_bytes,
                          void* workspace, size_t workspace_bytes, void* stream);
size_t     tlq_scale_search_gram_workspace_bytes(int64_t c_in, int64_t c_out, int32_t n_alpha,
                                                 const tlq_params* p);
tlq_status tlq_scale_search_gram(const void* gram, int64_t c_in,
                                 const void* W, int64_t c_out, int64_t ldw,
                                 const float* alpha_grid, int32_t n_alpha, const tlq_params* p,
                                 const float* x_stat /*[c_in]*/,
                                 float* best_scales /*[c_in]*/, int32_t* best_idx /*[1]*/,
                                 float* losses /*[n_alpha]*/, float* s_table_out /*[n_alpha,c_in] or NULL*/,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* ---- full-precision layer output (Sec. 3.2.1 f_fp without bias):
 * Y[t,o] = sum_c X[t,c] W[o,c], float accumulation, stored as yref_dtype. */
tlq_status tlq_ref_output(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                          const void* W, int64_t c_out, int64_t ldw,
                          void* Y, int64_t ldy, const tlq_params* p, void* stream);

/* ---- S6: quantisation-exposed propagation (Sec. 3.2.1 PassAct2):
 * X_next = f_q(X; s) = (X diag(s)^-1) Q_w(W diag(s))^T stored as x_dtype.
 * s: in float [c_in] (e.g. best_scales); X_next: out [n_tok, c_out]. */
size_t tlq_apply_best_workspace_bytes(int64_t n_tok, int64_t c_in, int64_t c_out,
                                      const tlq_params* p);
tlq_status tlq_apply_best(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx,
                          const void* W, int64_t c_out, int64_t ldw, const float* s,
                          const tlq_params* p, void* X_next, int64_t ld_next,
                          void* workspace, size_t workspace_bytes, void* stream);

/* ---- glue of the synthetic sequential chain (the workload's construction, not the paper's method):
 * builds the exposed input of the next linear from the quantised output of the
 * previous one (Sec. 3.2.1 PassAct2 propagation).
 *   v = Z (or Z*Zb elementwise when Zb != NULL);
 *   X_out[t,c] = round16( v[t,c] / sqrt(mean_c v[t,:]^2 + 1e-6) * m(t)[c] ),
 *   m(t) = m_a if period == 0 or (t mod period) < split, else m_b; NULL = ones.
 * Z, Zb, X_out: [n_tok, c] x_dtype; m_a, m_b: float [c].  float arithmetic. */
tlq_status tlq_rmsnorm_mul(const void* Z, int64_t n_tok, int64_t c, int64_t ldz, const void* Zb,
                           int64_t ldzb, const float* m_a, const float* m_b, int32_t period,
                           int32_t split, const tlq_params* p, void* X_out, int64_t ld_out,
                           void* stream);

/* ---- decoder-block glue for sequential calibration of a stack (Sec. 3.2.1:
 * activations are propagated through the model between two searches; the block
 * itself is the workload's, not the paper's).  All matrices are 16-bit
 * (p->x_dtype) device pointers, 16-byte aligned, row strides in elements and
 * multiples of 8; nothing is allocated; work is enqueued on `stream`.
 *
 * tlq_causal_attention: Out[t, h*128 .. h*128+127] =
 *   sum_{j <= t, same sample} softmax_j(q_t . k_j / sqrt(128)) v_j  per head h.
 * Rows are grouped in consecutive blocks of seq_len (one calibration sample
 * each); n_tok must be a multiple of seq_len.  head_dim must be 128
 * (TLQ_ERR_UNSUPPORTED otherwise).  Q, K, V may be column slices of one matrix.
 * Scores and the softmax are float; probabilities are rounded to x_dtype before
 * the second product; Out is rounded to x_dtype. */
tlq_status tlq_causal_attention(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V,
                                int64_t ldv, int64_t n_tok, int32_t n_heads, int32_t head_dim,
                                int32_t seq_len, const tlq_params* p, void* Out, int64_t ldo,
                                void* stream);
/* Out = G / (1 + exp(-G)) * U, elementwise in float, rounded to x_dtype; c % 8 == 0. */
tlq_status tlq_silu_mul(const void* G, int64_t ldg, const void* U, int64_t ldu, int64_t n_tok, int64_t c,
                        const tlq_params* p, void* Out, int64_t ldo, void* stream);
/* Out = H + Z, elementwise in float, rounded to x_dtype; Out may alias H or Z; c % 8 == 0. */
tlq_status tlq_residual_add(const void* H, int64_t ldh, const void* Z, int64_t ldz, int64_t n_tok,
                            int64_t c, const tlq_params* p, void* Out, int64_t ldo, void* stream);

/* ---- a decoder block that runs in 8 bits: what the searched setting act_bits <= 8, group = 0, symmetric = 1
 * (Sec. 4.1: per-token activations, per-channel symmetric weights) is searched for.  Forward only; forms for single
 * tokens and for whole prompts; no call synchronises, allocates or keeps anything, all can be captured into a graph.
 *
 * tlq_row_codes: rows to signed codes with one step a row, the quantiser of Q_a above and of Q_w with group = 0,
 * symmetric = 1 alike (float arithmetic, one rounding an operation, half to even):
 *   xt = x * factor[c];  step_r = max(max_c |xt|, 1e-5) / (2^(bits-1) - 1);
 *   code = clip(rint(xt / step_r), -2^(bits-1), 2^(bits-1) - 1).
 * X [n, c] x_dtype; factor: float [c], 16-byte aligned, or NULL (ones) - the searched scales for weight rows, their
 * reciprocals for tokens; bits 2..8; codes: out int8 [n, ldc], ldc (bytes) a multiple of 16 and at least c rounded up
 * to 128 (zeros are written behind c up to there, nothing beyond); 16-byte aligned; steps: out float [n]; n + 8 times the
 * smaller of 8 and c / 512 (rounded up) at most 2^29, here and in tlq_linear_i8.  A NaN has the
 * lowest code and no part in the step; an infinity makes the step infinite. */
tlq_status tlq_row_codes(const void* X, int64_t n, int64_t c, int64_t ldx, const float* factor, int32_t bits,
                         const tlq_params* p, int8_t* codes, int64_t ldc, float* steps, void* stream);
/* tlq_linear_i8: Y[t,o] = step_t * w_step[o] * sum_c code[t,c] * w_codes[o,c], with the codes and steps that
 * tlq_row_codes gives X (factor as there, bits = p->act_bits, TLQ_ERR_UNSUPPORTED if that is 0); the sums are exact.
 * w_codes int8 [c_out, ldw] and w_steps float [c_out] as tlq_row_codes writes them (the zeros behind c_in up to the next
 * multiple of 128 are read; w_steps 16-byte aligned); c_in a multiple of 8, at most 65536; ldw < 2^22; c_out < 2^29.
 * Y [n_tok, c_out] yref_dtype, 16-byte aligned, ldy a multiple of 8 (4 for float).  Workspace from the query. */
size_t tlq_linear_i8_workspace_bytes(int64_t n_tok, int64_t c_in);
tlq_status tlq_linear_i8(const void* X, int64_t n_tok, int64_t c_in, int64_t ldx, const float* factor,
                         const int8_t* w_codes, int64_t c_out, int64_t ldw, const float* w_steps, const tlq_params* p,
                         void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);

/* tlq_qk_norm_rope: queries and keys normalised for each head (norm = 1; 0: not) and rotated by their position:
 *   u = x / sqrt(mean_d x^2 + eps) * w[d];  angle = pos[t] * inv_freq[i] (in double), i < rot / 2;
 *   (u_a, u_b) -> (u_a cos - u_b sin, u_b cos + u_a sin), (a, b) = (i, i + rot/2), or (2i, 2i+1) with interleaved = 1;
 * d >= rot is not rotated.  Float arithmetic, one rounding to x_dtype at the end.
 * Q [n_tok, n_heads * head_dim], K [n_tok, n_kv_heads * head_dim] x_dtype, n_tok <= 2^26 - 4, 16-byte aligned, strides multiples of 8
 * (both may be column slices of one matrix); head_dim 64, 128 or 256 (TLQ_ERR_UNSUPPORTED otherwise); rot a multiple
 * of 16, 0 <= rot <= head_dim; eps >= 0 (with 0 a head of zeros gives NaN); pos int32 [n_tok] (any sign), inv_freq
 * double [rot/2]; wq, wk float [head_dim], 16-byte aligned, or NULL (ones; both have to be NULL without norm).  Q_out may be Q with the same stride, K_out likewise K; no
 * other overlap. */
tlq_status tlq_qk_norm_rope(const void* Q, int64_t ldq, int32_t n_heads, const void* K, int64_t ldk, int32_t n_kv_heads,
                            int64_t n_tok, int32_t head_dim, int32_t rot, int32_t interleaved, int32_t norm, float eps,
                            const float* wq, const float* wk, const int32_t* pos, const double* inv_freq,
                            const tlq_params* p, void* Q_out, int64_t ldqo, void* K_out, int64_t ldko, void* stream);

/* ---- keys and values of earlier tokens in 8 bits, in pages of `page` tokens with one step for each page and head.
 * A cache is a pool of n_pages pages for n_kv_heads heads:
 *   k int8 [n_pages, n_kv_heads, page, head_dim], k_step float [n_pages, n_kv_heads]: key = code * step;
 *   v int8 [n_pages, n_kv_heads, head_dim, page] (the tokens of a channel are contiguous), v_step likewise.
 * k and v 16-byte aligned; head_dim 64 or 128, page 16, 32, 64, 128 or 256 (TLQ_ERR_UNSUPPORTED otherwise).
 * A batch is n_seq sequences whose lengths live on the device: sequence s has lens[s] tokens, the newest of which are the
 * rows cu_new[s] .. cu_new[s+1]-1 of the call's matrices (cu_new int32 [n_seq + 1], ascending from 0; rows behind the last
 * sequence are neither read nor written); token j of it lives in page table[s * ld_table + j / page], j < max_pages * page.
 * max_new and max_len are upper bounds of a sequence's new tokens and of its length; launches are sized by them.
 * Device values are never trusted with an address: an entry of the table outside [0, n_pages) stands for a page of tokens
 * that do not exist (nothing is written, no query sees them), cu_new is held to [0, n_tok], new tokens beyond lens[s],
 * beyond the table or beyond the bounds are left out (the rows of Out behind a sequence's first max_new are then not written).
 * Bounds far above the real lengths cost speed: the keys are split by max_len. */
typedef struct tlq_kv_cache {
  uint32_t struct_size; /* = sizeof(tlq_kv_cache) */
  int32_t n_kv_heads, head_dim, page;
  int64_t n_pages;
  int8_t* k; float* k_step;
  int8_t* v; float* v_step;
} tlq_kv_cache;
typedef struct tlq_kv_batch {
  uint32_t struct_size; /* = sizeof(tlq_kv_batch) */
  int32_t n_seq;        /* 1 .. 65535 */
  const int32_t* cu_new; const int32_t* lens; const int32_t* table;
  int64_t ld_table;     /* entries between the table's rows, >= max_pages */
  int32_t max_pages, max_new, max_len;
  int32_t reserved;     /* 0 */
} tlq_kv_batch;
/* tlq_kv_append: the new tokens' keys and values as codes.  For a page and head, over its new tokens (float arithmetic):
 *   step = max(max |x|, 1e-5) / 127, and at least the page's step if it held tokens of the sequence before;
 *   code = clip(rint(x / step), -127, 127); codes held before: rint(code * (old step / step)).
 * Infinities count as +-127 and NaN as 0, neither has a part in the step.  Codes behind a sequence's last token stay
 * as they were.  K, V [n_tok, n_kv_heads * head_dim] x_dtype, 16-byte aligned, strides multiples of 8.  Sequences may
 * share pages that the call does not write; a page that two entries of the table name and give new tokens ends up undefined.
 * n_seq times the pages that max_new tokens can lie in: below 2^24. */
tlq_status tlq_kv_append(const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t n_tok, const tlq_kv_batch* b,
                         const tlq_kv_cache* c, const tlq_params* p, void* stream);
/* tlq_kv_attention: Out[r, h] = sum_{j <= pos(r)} softmax_j(scale * q_r . key_j) value_j, head h with the keys of head
 * h / (n_heads / n_kv_heads); row r of sequence s is its token pos(r) = lens[s] - (cu_new[s+1] - cu_new[s]) + r - cu_new[s].
 * scale: any finite number, 0 = 1 / sqrt(head_dim).  A row that sees no token gives zeros; a query that is not finite
 * makes NaN of its own row and head and of no other.  Scores, softmax and sums are
 * float; the matrix products take codes as they are, queries exactly (bf16 ones times a power of two of their row; channels
 * below 2^-31 of its largest are rounded to 2^-39 of it) and
 * probabilities times the page's step in fp16, which the softmax's sum takes as well unless a page's step lies so far below the
 * others' that halves would lose its keys (their weights are then summed as floats); Out is rounded to x_dtype.  Steps have to
 * be positive and finite in pages that a row sees (others may hold anything), and scores below 2^21 in size (beyond, a float holds them to a quarter at best); other rows are undefined.
 * Q, Out [n_tok, n_heads * head_dim] x_dtype, 16-byte aligned, strides multiples of 8; n_heads a multiple of n_kv_heads;
 * n_tok * (n_heads / n_kv_heads) and n_seq * n_kv_heads below 2^31 - 256, max_new * (n_heads / n_kv_heads) below 2^28,
 * that over 128 (rounded up) times n_seq * n_kv_heads below 2^30.
 * The workspace query reads sizes only, no pointer; the result does not depend on the workspace's contents. */
size_t tlq_kv_attention_workspace_bytes(int64_t n_tok, int32_t n_heads, const tlq_kv_batch* b, const tlq_kv_cache* c);
tlq_status tlq_kv_attention(const void* Q, int64_t ldq, int64_t n_tok, int32_t n_heads, float scale, const tlq_kv_batch* b,
                            const tlq_kv_cache* c, const tlq_params* p, void* Out, int64_t ldo, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ---- the block's other calls in low bits: what stands between its products, products of codes that are there already,
 * positions of images and video, and a cache in 4 bits.  Forward only; forms for single tokens and for whole prompts; no call
 * synchronises, allocates or keeps anything, all can be captured into a graph.
 *
 * tlq_add_norm_codes: the residual's addition, a root-mean-square norm and the codes of the normalised rows in one pass:
 *   h = round16(H + Z) (Z NULL: h = H);  r = float(1 / sqrt(mean_c h^2 + eps)) with the mean and the root in double;
 *   u = (h * r) * w[c];  step = max(max_c |u|, 1e-5) / (2^(bits-1) - 1);  code = clip(rint(u / step), -2^(bits-1), 2^(bits-1) - 1)
 * (float arithmetic, one rounding an operation, half to even; the double sum is off by 2^-46 at most, so that r is this float but in a row
 * of some millions, whose r may be its neighbour).  The
 * norm's weight and the searched scales' reciprocals are one factor w: float [c], 16-byte aligned, or NULL (ones).
 * H, Z, H_out [n, c] x_dtype, 16-byte aligned, strides multiples of 8; H_out may be NULL (not wanted), or H or Z with the same
 * stride; no other overlap.  c a multiple of 8, at most 65536; bits 2..8; eps >= 0 (with 0 a row of zeros gives NaN).  codes, ldc and steps as
 * in tlq_row_codes.  A row with h or r that is not finite (a mean and eps of 0, or near it) has a NaN step (and with it every
 * product of the row) and undefined codes.  n at most 2^21. */
tlq_status tlq_add_norm_codes(const void* H, int64_t ldh, const void* Z, int64_t ldz, int64_t n, int64_t c, const float* w,
                              float eps, int32_t bits, const tlq_params* p, void* H_out, int64_t ldho, int8_t* codes,
                              int64_t ldc, float* steps, void* stream);

/* tlq_linear_codes: tlq_linear_i8 on codes and steps that are there (tlq_add_norm_codes, tlq_row_codes), with an epilogue:
 *   y = act(step_t * w_step[o] * sum_c code[t,c] * w_codes[o,c] + bias[o]);  Y[t,o] = y + R[t,o], or y * R[t,o] with mul = 1.
 * codes int8 [n_tok, ldx] and w_codes with zeros behind c_in up to the next multiple of 128, 16-byte aligned, strides (bytes)
 * multiples of 16 and below 2^22; steps float [n_tok].  bias: float [c_out], 16-byte aligned, or NULL.  act: one of tlq_act.
 * R [n_tok, c_out] yref_dtype, aligned as Y, or NULL (mul has to be 0 then); Y may be R with the same stride; no other
 * overlap.  Float arithmetic, one rounding to yref_dtype at the end; NaN and +infinity pass an activation, -infinity may give NaN.  c_in, c_out, w_steps, Y as in tlq_linear_i8; of p the
 * type of Y is read.  Workspace from the query. */
typedef enum {
  TLQ_ACT_NONE = 0,
  TLQ_ACT_SILU = 1,       /* v / (1 + exp(-v)) */
  TLQ_ACT_GELU_TANH = 2,  /* v / 2 (1 + tanh(sqrt(2 / pi) (v + 0.044715 v^3))) */
  TLQ_ACT_GELU_ERF = 3    /* v / 2 (1 + erf(v / sqrt(2))) */
} tlq_act;
size_t tlq_linear_codes_workspace_bytes(int64_t n_tok, int64_t c_in);
tlq_status tlq_linear_codes(const int8_t* codes, int64_t ldx, const float* steps, int64_t n_tok, int64_t c_in, const int8_t* w_codes,
                            int64_t c_out, int64_t ldw, const float* w_steps, const float* bias, int32_t act, const void* R,
                            int64_t ldr, int32_t mul, const tlq_params* p, void* Y, int64_t ldy, void* workspace,
                            size_t workspace_bytes, void* stream);

/* tlq_qk_norm_rope_axes: tlq_qk_norm_rope with a position for each of n_axes axes (1..4; time, height and width of image and
 * video patches):  angle of frequency i = pos[axis[i] * ld_pos + t] * inv_freq[i].  pos int32 [n_axes, ld_pos], ld_pos >= n_tok; axis
 * int32 [rot/2] on the device, its values are held to [0, n_axes).  Everything else as there, and the same bits where a
 * token's positions agree. */
tlq_status tlq_qk_norm_rope_axes(const void* Q, int64_t ldq, int32_t n_heads, const void* K, int64_t ldk, int32_t n_kv_heads,
                                 int64_t n_tok, int32_t head_dim, int32_t rot, int32_t interleaved, int32_t norm, float eps,
                                 const float* wq, const float* wk, const int32_t* pos, int64_t ld_pos, int32_t n_axes,
                                 const int32_t* axis, const double* inv_freq, const tlq_params* p, void* Q_out, int64_t ldqo,
                                 void* K_out, int64_t ldko, void* stream);

/* ---- a cache in 4 bits: pages as above, with a step for each token, head and 32 channels (4.5 bits a value), so that a token's
 * codes hang on nothing but the token and never change once they are written, however the tokens are dealt to calls.
 * Codes are words of eight: element e of a word lies in the four bits from 4 (e / 2) + 16 (e % 2) up, as code + 8.
 *   k uint32 [n_pages, n_kv_heads, page, head_dim / 8];  k_step half [n_pages, n_kv_heads, page, head_dim / 32];
 *   v uint32 [n_pages, n_kv_heads, head_dim, page / 8] (the tokens of a channel are contiguous);
 *   v_step half [n_pages, n_kv_heads, head_dim / 32, page];   key and value = (nibble - 8) * step, which halves hold
 * exactly (appends write nibbles 1..15 and steps up to 9344; a nibble of 0 beside a step above 8188 would be none).
 * All four 16-byte aligned; head_dim and page as above.  Batches are the same tlq_kv_batch, and device values as little trusted. */
typedef struct tlq_kv4_cache {
  uint32_t struct_size; /* = sizeof(tlq_kv4_cache) */
  int32_t n_kv_heads, head_dim, page;
  int64_t n_pages;
  uint32_t* k; uint16_t* k_step;
  uint32_t* v; uint16_t* v_step;
} tlq_kv4_cache;
/* tlq_kv4_append: the new tokens' keys and values as codes.  For a token, head and 32 neighbouring channels (float arithmetic):
 *   step = max(max |x|, 1e-5) / 7 rounded to bf16 and then to half (its 8 significant bits keep code * step exact), 9344 at most;
 *   code = clip(rint(x / step), -7, 7).
 * Infinities count as +-7 and NaN as 0, neither has a part in the step.  Everything that is not a new token's stays as it was.
 * K, V and pages that are shared as in tlq_kv_append.  Here and in tlq_kv4_read, with e = (min(max_new, n_tok) + 14) / 8 rounded down
 * and both quotients rounded up, n_seq (n_kv_heads (e head_dim / 512) / 4) is below 2^23. */
tlq_status tlq_kv4_append(const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t n_tok, const tlq_kv_batch* b,
                          const tlq_kv4_cache* c, const tlq_params* p, void* stream);
/* tlq_kv4_read: what the tokens of a batch's rows stand for: row r of K_out and V_out [n_tok, n_kv_heads * head_dim] x_dtype, 16-byte aligned, strides
 * multiples of 8, is the token that a tlq_kv4_append of the same batch writes from row r (cu_new from whole lengths reads whole
 * sequences).  Rows before a sequence's first token, beyond its bounds or in a page that there is not give zeros; rows behind
 * the last sequence, or behind a sequence's first max_new, are not written.  Exact in half, rounded to bf16.  K_out or V_out may be NULL. */
tlq_status tlq_kv4_read(const tlq_kv_batch* b, const tlq_kv4_cache* c, const tlq_params* p, int64_t n_tok, void* K_out, int64_t ldk,
                        void* V_out, int64_t ldv, void* stream);
/* tlq_kv4_attention: tlq_kv_attention over a cache in 4 bits: the same rows, masks, limits and workspace rules.  Keys and values
 * enter the matrix products exactly, queries as there, and softmax weights rounded to halves, which the softmax's sum takes as well; scores,
 * softmax and sums are float.  Scores may have any size here: beyond 2^24 they are rounded to floats before the exponential, and where
 * floats end the largest takes all of the weight.  Steps have to be finite in tokens that a row sees; others may hold anything. */
size_t tlq_kv4_attention_workspace_bytes(int64_t n_tok, int32_t n_heads, const tlq_kv_batch* b, const tlq_kv4_cache* c);
tlq_status tlq_kv4_attention(const void* Q, int64_t ldq, int64_t n_tok, int32_t n_heads, float scale, const tlq_kv_batch* b,
                             const tlq_kv4_cache* c, const tlq_params* p, void* Out, int64_t ldo, void* workspace,
                             size_t workspace_bytes, void* stream);

/* ---- host-side self check (no GPU work, no device memory): walks the block -> tile map that
 * the contraction kernels (S3/S4, f_fp, S6) would use for this problem shape, in both of its
 * orders (candidates inside every patch row / candidate-outermost), both patch shapes and all tile
 * sizes (128 x 128 outputs, and 256 outputs x 192, 256 or 320 tokens), the quadratic form's and the
 * symmetric products' maps, and returns how many (candidate, output tile) pairs are NOT produced exactly
 * once - 0 for correct maps, -1 for an invalid shape.  *blocks (may be NULL) receives the number of
 * workgroups of the launch that the library makes for the shape, with the tile size that it picks: with one
 * candidate the product of tlq_ref_output and tlq_apply_best, with several the contraction of a search in
 * 4 bits without activation codes. */
int64_t tlq_selftest_tile_map(int64_t n_tok, int64_t c_in, int64_t c_out, int32_t n_cand,
                              int64_t* blocks);

/* ---- optional per-kernel timing (host-side bookkeeping only).
 * While enabled, every kernel the library launches is bracketed by HIP events
 * on the launch stream.  tlq_profile_collect waits for the recorded events
 * and folds them into per-kernel totals; tlq_profile_get reads entry i:
 * kernel name, number of launches, total milliseconds, and the total
 * algorithmic work (flops for the contraction kernels, bytes otherwise). */
tlq_status tlq_profile_enable(int on);
int tlq_profile_enabled(void);
tlq_status tlq_profile_reset(void);
tlq_status tlq_profile_collect(void);
int tlq_profile_count(void);
tlq_status tlq_profile_get(int i, char* name, size_t name_cap, int64_t* launches,
                           double* total_ms, double* total_work);

#ifdef __cplusplus
}
#endif
#endif /* TLQ_H */
