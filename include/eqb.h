/*
 * eqb.h -- C ABI of libeqb.so: the per-layer MoE routing-balance path of
 * Exact Quantile Balancing (EQB) and Load-Error Injection (LEI),
 * arXiv 2609.28053, on one NVIDIA GB300 (sm_103a), and the operators of a
 * router's training step beside it: the balance loss with its gradient, the
 * projection's gradients, and AdamW; and of the experts behind the router: the
 * gate's weights, the experts' rows, 8-bit values with block scales, the
 * grouped products and the weighted sum back.
 *
 * Notation follows the paper: T tokens, E routed experts, K experts per
 * token, router logits z[T,E], expert bias b[E], cutoff tau_t = the (K+1)st
 * largest entry of z_t + b, expert loads f_e, target rank r = TK/E.
 *
 * Conventions shared by every call
 * --------------------------------
 *  - Pointers named as device buffers are CUDA device (or managed) pointers
 *    that the caller allocates and owns.  Unless a function says otherwise,
 *    the library allocates no device memory and keeps no state between calls.
 *  - `stream` is a cudaStream_t passed as void* (NULL = legacy default
 *    stream).  Every call only enqueues work on it and returns without
 *    synchronising; results are valid once the stream has reached them.
 *  - Row-major layouts with the expert index fastest: z[t*E + e].
 *  - bf16 values travel as their raw 16-bit patterns (eqb_bf16).
 *  - Outputs documented as "+=" are accumulated into; the caller zeroes them
 *    first.  This is what lets token partitions (the data-parallel ranks of
 *    Algorithm 1, here slices of one batch) be summed in device memory, and
 *    lets a multi-GPU caller insert its own all-reduce between passes.
 *  - Return value: an eqb_status.  Arguments are validated on the host
 *    before anything is launched; an invalid call launches nothing.
 *    EQB_ERR_CUDA reports a launch failure (cudaGetLastError after launch).
 *  - Errors found by the device (non-finite data, an unreachable rank) are
 *    written to the optional device word `err_flag` (int32, nullable) as the
 *    eqb_status code; the caller zeroes it before the call and reads it after
 *    synchronising.  Outputs of a call that flagged an error are unspecified.
 *  - Microbatches (the paper's local batches B_l, Sec. 2) are contiguous
 *    token ranges given by device int64 offsets[M+1]: offsets[0] = 0,
 *    offsets[M] = T, non-decreasing (empty microbatches are allowed).
 *    The library reads them on the device; they are not checked on the host.
 *  - Supported sizes: 1 <= K, K + 1 <= 32, K < E, E a multiple of 8 with
 *    E <= 1024, T <= 2^31 - 2^24.  T = 0 is a valid no-op for the streaming
 *    calls.
 *  - Device buffers of bf16 logits must be 16-byte aligned; fp32 gradient
 *    buffers 16-byte aligned.  Misaligned pointers give EQB_ERR_INVALID_ARG.
 */
#ifndef EQB_H
#define EQB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef uint16_t eqb_bf16; /* raw bf16 bit pattern */

typedef enum eqb_status {
  EQB_OK = 0,
  EQB_ERR_INVALID_ARG = 1, /* host-side validation failed; nothing launched */
  EQB_ERR_UNSUPPORTED = 2, /* valid by the paper, outside the sizes the library supports */
  EQB_ERR_CUDA = 3,        /* a CUDA launch or runtime call failed */
  EQB_ERR_NONFINITE = 4,   /* device flag: non-finite z, b or score, a margin
                              of magnitude >= 2^127, or a moment of AdamW */
  EQB_ERR_RANK = 5         /* device flag: a histogram holds fewer than r
                              margins for some expert */
} eqb_status;

/* Human-readable name of a status code (static string). */
const char *eqb_status_string(int status);

/* Library version as MAJOR*10000 + MINOR*100 + PATCH. */
int eqb_version(void);

/* Target rank r = ceil(T*K / E) (Sec. 3: r = TK/E, assumed integral by the
 * paper; rounded up otherwise, the inverse-CDF quantile).  Returns -1 for
 * invalid arguments.  Host only. */
int64_t eqb_target_rank(int64_t T, int32_t E, int32_t K);

/* Routing and the coarse EQB pass.  Sec. 2 (Eq. 1 and the QB paragraph),
 * Algorithm 1 step 1.
 *
 * For each token t: s_e = fp32(z_{t,e}) + b_e (fp32, round to nearest
 * even); the top-K set of s (ties to the lower expert index), written to
 * topk_idx[t, 0..K-1] in descending score order; tau[t] = the (K+1)st
 * largest s (fp32).  loads[l, e] += number of tokens of microbatch l whose
 * top-K set contains e.
 *
 * hist_hi (nullable): when given, also accumulates Algorithm 1's coarse
 * histogram: for every (t, e), the margin m = bf16_rne(tau_t - fp32(z_{t,e}))
 * is encoded by the order-preserving key kappa(m) (bf16 pattern x ->
 * x & 0x8000 ? ~x : x | 0x8000, 16 bits) and hist_hi[e, kappa(m) >> 8] += 1.
 *
 *   z         device bf16 [T,E], 16-byte aligned          (in)
 *   b         device fp32 [E]                              (in)
 *   mb_offsets device int64 [M+1] (nullable iff loads is NULL)
 *   topk_idx  device int32 [T,K]   (nullable)              (out)
 *   tau       device fp32 [T]                              (out)
 *   loads     device int32 [M,E] += (nullable)             (in/out)
 *   hist_hi   device int32 [E,256] += (nullable)           (in/out)
 *   err_flag  device int32 (nullable): EQB_ERR_NONFINITE for a non-finite
 *             b_e or NaN score, or (with hist_hi) a non-finite margin.
 *
 * With hist_hi the coarse pass runs as a second kernel over z (on GB300 the
 * two kernels are faster than the one-read eqb_route_hist_fused).
 */
eqb_status eqb_route_topk(const eqb_bf16 *z, const float *b, int64_t T, int32_t E,
                          int32_t K, const int64_t *mb_offsets, int32_t M,
                          int32_t *topk_idx, float *tau, int32_t *loads,
                          int32_t *hist_hi, int32_t *err_flag, void *stream);

/* Routing and the coarse pass in one pass over z (Sec. 2 Eq. 1 and the QB
 * paragraph; Algorithm 1 step 1): the results of eqb_route_topk with hist_hi,
 * from one kernel that routes each 32-token tile staged in shared memory and
 * then counts the same staged tile, so z is read from DRAM once instead of
 * twice.  E = 128 or 256 and K + 1 <= 16, else EQB_ERR_UNSUPPORTED.
 * Arguments as in eqb_route_topk; hist_hi is required.  Bit-identical
 * outputs; slower than the two kernels on GB300, although they read z twice:
 * beside the routing tiles the counting has a third of the coarse pass's warps
 * and a window of bins that takes more instructions. */
eqb_status eqb_route_hist_fused(const eqb_bf16 *z, const float *b, int64_t T, int32_t E,
                                int32_t K, const int64_t *mb_offsets, int32_t M,
                                int32_t *topk_idx, float *tau, int32_t *loads,
                                int32_t *hist_hi, int32_t *err_flag, void *stream);

/* Coarse pass on its own (Algorithm 1 step 1): recomputes the margins from z
 * and tau and accumulates hist_hi[e, kappa(m) >> 8] += 1 over T tokens.
 * Margins of magnitude >= 2^127 or non-finite set EQB_ERR_NONFINITE: kappa
 * gives them the high bytes 0x00 and 0xff, which the method's domain
 * (|m| < 2^127) leaves out. */
eqb_status eqb_margin_hist_pass1(const eqb_bf16 *z, const float *tau, int64_t T,
                                 int32_t E, int32_t *hist_hi, int32_t *err_flag,
                                 void *stream);

/* Fine pass (Algorithm 1 step 4; Sec. 3 "the second pass simply rescans
 * local margins whose high byte matches the selected bin"): recomputes
 * every margin from z and tau and, where kappa(m) >> 8 == u[e], accumulates
 * hist_lo[e, kappa(m) & 0xff] += 1.  No margin array is materialised.
 *   u        device uint8 [E] (from eqb_select_quantile pass 1)
 *   hist_lo  device int32 [E,256] += */
eqb_status eqb_margin_hist_pass2(const eqb_bf16 *z, const float *tau, int64_t T,
                                 int32_t E, const uint8_t *u, int32_t *hist_lo,
                                 void *stream);

/* Selection on a summed histogram (Algorithm 1 steps 3, 5 and 6).
 *   pass 1: reads hist = H [E,256]; writes u[e] = min{u : sum_{j<=u} H[e,j]
 *           >= r} and rho[e] = r - sum_{j<u_e} H[e,j].  r is the global
 *           target rank (eqb_target_rank of the whole batch).  Sets
 *           EQB_ERR_NONFINITE if a margin landed in high byte 0x00 or 0xff
 *           (magnitude >= 2^127 or non-finite) and EQB_ERR_RANK if H[e,:]
 *           sums to less than r.
 *   pass 2: reads hist = L [E,256], u and rho; writes v_e = min{v :
 *           sum_{j<=v} L[e,j] >= rho_e} and q_hat[e] = kappa^{-1}((u_e << 8)
 *           | v_e), the exact r-th smallest margin (a zero as +0).
 *   q_hat is ignored in pass 1; r is ignored in pass 2. */
eqb_status eqb_select_quantile(const int32_t *hist, int32_t E, int32_t pass,
                               int64_t r, uint8_t *u, int32_t *rho, eqb_bf16 *q_hat,
                               int32_t *err_flag, void *stream);

/* Bias update of Eq. (2): b_next[e] = (float)((double)q_hat[e] - mean) with
 * mean = (sum over e = 0..E-1 in ascending order, in fp64) / E.  The fixed
 * order makes the result bit-reproducible.  b_next is used for routing in
 * the next optimizer step. */
eqb_status eqb_bias_update(const eqb_bf16 *q_hat, int32_t E, float *b_next,
                           void *stream);

/* Load-Error Injection, Sec. 4 Eq. (LEI) with the normalisation Eq. (norm).
 * For each microbatch l with n_l tokens (empty ones are skipped):
 *   rho_e = f_{l,e} / (K n_l / E) - 1;
 *   c > 0:  xi = max_e |rho_e| / c,  sigma = tanh(xi) / xi (1 at xi = 0);
 *   c <= 0: sigma = 1 (unnormalised LEI);
 *   grad_s[t, e] += eta * sigma * rho_e for every t in the microbatch and
 *   every expert e.  rho and the product eta * sigma * rho are formed in
 *   fp64 (sigma in fp32, within a few fp32 ulps of tanh(xi) / xi), rounded
 *   to fp32, and added in fp32.
 *   grad_s  device fp32 [T,E], 16-byte aligned, updated in place
 *   loads   device int32 [M,E] (the local loads from eqb_route_topk) */
eqb_status lei_inject_grad(float *grad_s, const int32_t *loads,
                           const int64_t *mb_offsets, int32_t M, int64_t T,
                           int32_t E, int32_t K, float eta, float c, void *stream);

/* The Load-Error Injection coefficients (Sec. 4, Eqs. LEI and norm) as a
 * table: coef[l, e] = (float)(eta * sigma_l * rho_{l,e}), rho and sigma of
 * microbatch l as in lei_inject_grad, by the same arithmetic (so the same
 * bits as the coefficient lei_inject_grad adds).  An empty microbatch
 * gets a row of zeros.
 *   loads  device int32 [M,E]                          (in)
 *   coef   device fp32 [M,E], 16-byte aligned          (out) */
eqb_status lei_coefficients(const int32_t *loads, const int64_t *mb_offsets,
                            int32_t M, int32_t E, int32_t K, float eta, float c,
                            float *coef, void *stream);

/* A histogram pass of Algorithm 1 with part of Load-Error Injection streamed
 * beside it, in one kernel: pass 1 is eqb_margin_hist_pass1 (hist = hist_hi,
 * err_flag used, u ignored), pass 2 is eqb_margin_hist_pass2 (hist =
 * hist_lo, u required, err_flag ignored), and for the tokens t in
 * [lei_t0, lei_t1) every grad_s[t, e] += coef[l(t), e] in fp32, l(t) the
 * microbatch of t (Sec. 4, Eq. LEI).  The counting takes issue slots beside its
 * reads and the injection is a DRAM stream, so the two share the GPU better
 * than back to back.
 * Results are bit-identical to the separate calls; the one-call step runs
 * pass 2 with all of the tokens.
 *   grad_s  device fp32 [T,E], 16-byte aligned, updated in place on [lei_t0, lei_t1)
 *   coef    device fp32 [M,E] from lei_coefficients, 16-byte aligned
 *   0 <= lei_t0 <= lei_t1 <= T, else EQB_ERR_INVALID_ARG. */
eqb_status eqb_margin_hist_lei(const eqb_bf16 *z, const float *tau, int64_t T,
                               int32_t E, int32_t pass, const uint8_t *u,
                               int32_t *hist, int32_t *err_flag, float *grad_s,
                               const float *coef, const int64_t *mb_offsets,
                               int32_t M, int64_t lei_t0, int64_t lei_t1,
                               void *stream);

/* Bytes of device workspace eqb_layer_step needs for E experts (the two
 * [E,256] histograms, block counters, u, rho, q_hat and a 65,536-float
 * LEI coefficient table, each 256-byte aligned; 788,480 bytes for
 * E = 256). */
size_t eqb_layer_workspace_bytes(int32_t E);

/* One layer's whole routing-balance step in one call, in the paper's order:
 * routing (Sec. 2), Algorithm 1's coarse pass, selection, fine pass,
 * selection, the Eq. (2) bias update, then Load-Error Injection (Sec. 4,
 * Eqs. LEI and norm) on grad_s when grad_s is given.  Results are identical
 * to the individual calls above.  When M * E <= 65,536 the injection is
 * streamed by the fine pass (eqb_margin_hist_lei), with the coefficients
 * formed beside the coarse pass; otherwise LEI runs last (lei_inject_grad).
 * The selections (eqb_select_quantile) and eqb_bias_update run inside the
 * fine pass.
 *   z, b, mb_offsets, M, topk_idx (nullable), tau, eta, c: as in
 *             eqb_route_topk / lei_inject_grad;
 *   mb_offsets_host host copy of mb_offsets (nullable; validated when given)
 *   r         global target rank; r <= 0 means eqb_target_rank(T, E, K)
 *   loads     device int32 [M,E], overwritten (zeroed by the call)
 *   b_next    device fp32 [E] (out): the bias for the next step
 *   grad_s    device fp32 [T,E] updated in place, or NULL (no LEI)
 *   workspace device buffer of at least eqb_layer_workspace_bytes(E) bytes,
 *             256-byte aligned, owned by the caller; its contents on return
 *             are the step's histograms and selections
 * Histograms are local to the call, so this entry point is for a single
 * process; a multi-GPU caller all-reduces between the per-pass calls. */
eqb_status eqb_layer_step(const eqb_bf16 *z, const float *b, int64_t T, int32_t E, int32_t K,
                          const int64_t *mb_offsets, const int64_t *mb_offsets_host, int32_t M,
                          int64_t r, int32_t *topk_idx, float *tau, int32_t *loads, float *b_next,
                          float *grad_s, float eta, float c, void *workspace,
                          size_t workspace_bytes, int32_t *err_flag, void *stream);

/* eqb_layer_step for callers that cannot allocate device memory (no
 * counterpart in the paper; a library convenience).  Plugins hosted by a
 * framework or server that owns all device memory through its own pool, and
 * code that must not stall on or fail at an allocation, can call this
 * instead: it takes the same inputs and outputs but no workspace, and uses a
 * scratch array compiled into the library.
 *   - The scratch is eqb_layer_workspace_bytes(256) = 788,480 bytes: the
 *     step's two histograms, block counters, u, rho, q_hat and the
 *     65,536-float LEI coefficient table, enough for E <= 256; E > 256 returns
 *     EQB_ERR_UNSUPPORTED.  Every GPU that loads the library keeps
 *     this array until the process exits.
 *   - The first call on each device looks up the array's device address
 *     (cudaGetSymbolAddress) with that device current; make it before any
 *     stream capture.  It allocates nothing.  The address is kept for the
 *     life of the process: after cudaDeviceReset on that device it is stale,
 *     and calls must not be made there again.
 *   - All calls on a device share the array, which keeps the previous
 *     call's contents (the step zeroes the histograms before counting);
 *     calls that overlap on the GPU race on it.
 * Arguments and results are those of eqb_layer_step. */
eqb_status eqb_layer_step_noalloc(const eqb_bf16 *z, const float *b, int64_t T, int32_t E,
                                  int32_t K, const int64_t *mb_offsets,
                                  const int64_t *mb_offsets_host, int32_t M, int64_t r,
                                  int32_t *topk_idx, float *tau, int32_t *loads, float *b_next,
                                  float *grad_s, float eta, float c, int32_t *err_flag,
                                  void *stream);

/* Router logits, Sec. 2 (Eq. 1: z_t = W_r x_t):
 *   z[t, e] = bf16_rne(sum_k x[t, k] * W_r[e, k]),
 * bf16 inputs, fp32 accumulation on the tensor cores (tcgen05, accumulators
 * in tensor memory).  The accumulation order is the hardware's, so an entry
 * can differ from the exactly rounded value by one bf16 ulp plus the fp32
 * accumulation error.
 * The order also depends on how many tokens share the call.  With d >= 1,024
 * the columns are summed in eight parts up to T = 1,024, in four up to 4,224
 * and in two up to 8,448 (there from d = 3,072 on at E = 64, from 1,536 on at
 * other E <= 128), and the parts then added in order; otherwise in one sum
 * (the limits are those of 152 SMs).  So a token's z, and at near ties its
 * experts, can differ by a bf16 rounding between calls of different T.  The
 * same call on the same inputs gives the same bits; no order is further from
 * the exact sums than the one sum.
 *   x        device bf16 [T, d] row-major, 16-byte aligned     (in)
 *   W_r      device bf16 [E, d] row-major, 16-byte aligned     (in)
 *   z        device bf16 [T, E] row-major, 16-byte aligned     (out)
 *   err_flag device int32 (nullable): EQB_ERR_CUDA if the kernel's pipeline
 *            stalled and it gave up waiting (no result is then valid).
 * Supported: d a positive multiple of 64, E a multiple of 16 with
 * 16 <= E <= 256, 0 <= T <= 2^31 - 2^24.  One block per SM, which takes all of
 * the SM's tensor memory (half of it where the columns are summed in parts). */
eqb_status eqb_router_logits(const eqb_bf16 *x, const eqb_bf16 *W_r, int64_t T, int32_t d,
                             int32_t E, eqb_bf16 *z, int32_t *err_flag, void *stream);

/* GShard auxiliary-loss gradient: the comparison injection beside LEI
 * (Sec. 2, the loss alpha sum_e F_e P^G_e with F stop-gradient; App. D,
 * Eq. (gshard-grad)).  For every token t of microbatch l (n_l tokens):
 *   s_e = sigmoid(fp32(z_{t,e})),  d_t = sum_e s_e,  p_e = s_e / d_t,
 *   R_e = f_{l,e} / (K n_l) - 1/E,
 *   grad_s[t, j] += alpha / (n_l d_t) * (R_j - sum_e p_e R_e).
 * R and alpha / n_l are formed in fp64 and rounded to fp32; the rest is fp32
 * (expf, sums over the token's experts, no fused multiply-add).
 *   grad_s     device fp32 [T,E], 16-byte aligned (in/out)
 *   z          device bf16 [T,E], 16-byte aligned (in): the unbiased logits
 *   loads      device int32 [M,E] (in), mb_offsets device int64 [M+1] (in):
 *              as in lei_inject_grad
 * Supported: E a multiple of 8, E <= 1024, 0 <= T <= 2^31 - 2^24. */
eqb_status gshard_inject_grad(float *grad_s, const eqb_bf16 *z, const int32_t *loads,
                              const int64_t *mb_offsets, int32_t M, int64_t T, int32_t E,
                              int32_t K, float alpha, void *stream);

/* The two estimates of the global quantile that Sec. 2 compares EQB with.
 * Both take the margins m = bf16_rne(tau_t - fp32(z_{t,e})) of
 * eqb_margin_hist_pass1 (so tau comes from eqb_route_topk), end with the
 * Eq. (2) centering b_e = fp32(x_e - mean(x)) (fp64, mean summed in ascending
 * expert order), and use a caller-provided workspace (256-byte aligned).
 * Supported: E a multiple of 8, E <= 1024, T >= 1.
 *
 * Rank-averaged QB: every shard p (token range [offsets[p], offsets[p+1]))
 * selects its own K/E quantile exactly (the r_p-th smallest margin,
 * r_p = ceil(n_p K / E), by the same two radix passes as EQB); x_e is the
 * mean over the non-empty shards of those quantiles (fp64, summed in
 * ascending shard order).  Its workspace is
 * eqb_rank_averaged_workspace_bytes(E, P) bytes (per-shard histograms).
 *   shard_offsets_host  host int64 [P+1], 0 = first <= ... <= last = T,
 *                       1 <= P <= 65535
 *   q_shards            device bf16 [P,E] (out): row p holds shard p's
 *                       quantiles (+0 for an empty shard)
 *   err_flag            as in eqb_select_quantile
 * The result depends on how the tokens are sharded; EQB's does not. */
size_t eqb_rank_averaged_workspace_bytes(int32_t E, int32_t P);
eqb_status eqb_rank_averaged_bias(const eqb_bf16 *z, const float *tau, int64_t T, int32_t E,
                                  int32_t K, const int64_t *shard_offsets_host, int32_t P,
                                  eqb_bf16 *q_shards, float *b_out, void *workspace,
                                  size_t workspace_bytes, int32_t *err_flag, void *stream);

/* Fixed-resolution histogram: 256 equal-width bins over all tokens, margin m
 * in bin j = floor(fp32(fp32(m - lo) * fp32(1 / width))) clamped to
 * [0, 255]; x_e = lo + (j_e + 1) * width (fp64), the upper edge of the first
 * bin whose cumulative count reaches r = ceil(T K / E).  Its resolution is
 * the bin width, the limitation EQB removes.  Its workspace is
 * eqb_layer_workspace_bytes(E) bytes.
 *   lo, width   finite, width > 0
 *   estimate    device double [E] (out, nullable): x before centering */
eqb_status eqb_fixed_hist_bias(const eqb_bf16 *z, const float *tau, int64_t T, int32_t E,
                               int32_t K, float lo, float width, float *b_out, double *estimate,
                               void *workspace, size_t workspace_bytes, int32_t *err_flag,
                               void *stream);

/* Balance metric MaxVio, Sec. 5 (Metrics) and App. E (balance metrics):
 *   MaxVio(B) = max_e [ f_e(B) / fbar(B) - 1 ],   fbar(B) = K |B| / E,
 * in fp64 (fbar formed as (K * |B|) / E, then one division and one
 * subtraction).
 *   maxvio[0]  Global MaxVio: the loads summed over the M microbatches,
 *              |B| = offsets[M] - offsets[0].
 *   maxvio[1]  Local MaxVio: the plain mean, summed in ascending order, of
 *              the per-microbatch values over the non-empty microbatches (an
 *              empty one has no fbar); 0 if every microbatch is empty.
 *   loads      device int32 [M,E] (in): per-microbatch loads, as written by
 *              eqb_route_topk or eqb_layer_step
 *   mb_offsets device int64 [M+1] (in): as in eqb_route_topk
 *   maxvio     device double [2] (out), 8-byte aligned
 *   per_mb     device double [M] (out, nullable): each microbatch's MaxVio,
 *              0 for an empty one
 * The paper reports the maximum over layers and a mean over steps; a caller
 * takes those across calls.  Supported: 1 <= M <= 16384. */
eqb_status eqb_maxvio(const int32_t *loads, const int64_t *mb_offsets, int32_t M, int32_t E,
                      int32_t K, double *maxvio, double *per_mb, void *stream);

/* Router logits and routing in one kernel, with the coarse pass in the same
 * kernel or after it: eqb_router_logits followed by eqb_route_topk.  Each token
 * is routed from the tensor-memory accumulator of its row, or, where the
 * columns are summed in parts, from the sum of its row, so z is written once
 * and not read back for routing.  The paper computes the same steps one after the other
 * (Sec. 2, Eq. 1, then top-K of s = z + b, then Algorithm 1 step 1); fusing
 * them is a property of this library.
 *   x, W_r, z   as in eqb_router_logits; z is still written (the fine pass
 *               and LEI read it)
 *   b, K, mb_offsets, M, topk_idx, tau, loads, hist_hi, err_flag
 *               as in eqb_route_topk: topk_idx [T,K] (nullable), tau [T],
 *               loads [M,E] += (nullable; then mb_offsets may be NULL),
 *               hist_hi [E,256] += (nullable): the coarse histogram, counted
 *               in the same kernel from the rows it just stored (read back
 *               from L2) when the columns are summed in one sum and no block of
 *               the kernel routes more than 65,535 tokens (T <= 65,408 x the SM
 *               count: 511 tiles of 128 rows per block), else by the coarse
 *               pass over z after it
 * The order of the sums is that of eqb_router_logits for the same T, d and E.
 * Results equal those of the calls made one after the other on the same
 * inputs, bit for bit.  err_flag: EQB_ERR_NONFINITE as in eqb_route_topk,
 * EQB_ERR_CUDA as in eqb_router_logits.
 * Supported: E in {64, 128}, 1 <= K <= 8, K < E, d a positive multiple of
 * 64, 0 <= T <= 2^31 - 2^24; other shapes return EQB_ERR_UNSUPPORTED (make
 * the two calls instead). */
eqb_status eqb_router_route(const eqb_bf16 *x, const eqb_bf16 *W_r, int64_t T, int32_t d,
                            int32_t E, int32_t K, const float *b, const int64_t *mb_offsets,
                            int32_t M, eqb_bf16 *z, int32_t *topk_idx, float *tau,
                            int32_t *loads, int32_t *hist_hi, int32_t *err_flag, void *stream);

/* The routing-balance step of one layer from the router input: the router
 * projection z = bf16(x W_r^T) (Sec. 2, Eq. 1) followed by everything
 * eqb_layer_step does.  For E in {64, 128} and K <= 8 the projection, the
 * routing and the coarse histogram run as one kernel (as eqb_router_route with
 * hist_hi), and the fine pass then streams all of LEI (when M * E <=
 * 65,536); otherwise the projection, then eqb_route_topk and the schedule
 * of eqb_layer_step.  The projection here always takes the columns in one sum,
 * whatever T is: where eqb_router_logits and eqb_router_route take them in
 * parts (few tokens), their z can differ from the step's by a bf16 rounding,
 * and the top-K at near ties with it.  The other steps are those of
 * eqb_layer_step, and so are the arguments from b on; z is an output here
 * (device bf16 [T,E], 16-byte aligned).
 *   x, W_r, d   as in eqb_router_logits.
 * Returns EQB_ERR_UNSUPPORTED for d not a multiple of 64, E not a multiple
 * of 16 or E > 256 (the projection's limits), beside eqb_layer_step's own
 * conditions. */
eqb_status eqb_router_layer_step(const eqb_bf16 *x, const eqb_bf16 *W_r, int64_t T, int32_t d,
                                 int32_t E, int32_t K, const float *b,
                                 const int64_t *mb_offsets, const int64_t *mb_offsets_host,
                                 int32_t M, int64_t r, eqb_bf16 *z, int32_t *topk_idx,
                                 float *tau, int32_t *loads, float *b_next, float *grad_s,
                                 float eta, float c, void *workspace, size_t workspace_bytes,
                                 int32_t *err_flag, void *stream);

/* Balance loss and per-expert counts, with the gradient (the auxiliary loss
 * alpha sum_e F_e P_e of Sec. 2 as a whole, where gshard_inject_grad adds the
 * gradient of one form of it).  For microbatch l with n valid tokens (all of
 * them, or those with a non-zero mask byte):
 *   f_{l,e} = entries of the valid tokens' lists that name expert e (an entry
 *             outside [0, E), such as -1, names none),  F_e = f_{l,e} / (K n),
 *   p_t     = softmax(z_t), or sigmoid(z_t) divided by its sum over the experts,
 *   loss[l] = (alpha sum_e F_e P_e,  zeta mean_t lse_t^2),
 *             P_e = mean_t p_{t,e}, lse_t = log sum_e exp(z_{t,e}),
 * and, F being a constant, the gradient of grad_scale * (the two summed over
 * the microbatches) with respect to z:
 *   d_{t,j} = p_j (alpha / n (F_j - sum_e p_e F_e) + 2 zeta / n lse_t)   (softmax)
 *   d_{t,j} = p_j (1 - s_j) alpha / n (F_j - sum_e p_e F_e)              (sigmoid)
 * written as grad_out = grad_in + d (grad_out = d without grad_in).  A token
 * that is masked out contributes nothing, its d is 0 and its row of z may hold
 * anything.  A logit of -inf closes its expert to the token (p = 0); a row that is
 * -inf throughout has p = 0, lse = 0 and d = 0 and still counts in n.  An empty
 * microbatch has loss 0 and P = 0.
 * The arithmetic is fp32 (p and lse; the exponentials within a few ulps).  F, and
 * for the gradient F - 1/E, come from whole numbers, f and f E - K n, by factors
 * rounded to fp32; sums over tokens are formed in a fixed order, of long
 * microbatches the last in fp64, so the same call gives the same bits.  The counts need no z, so one pass over it
 * gives loss and gradient.
 *   z          device bf16 [T,E], or fp32 with z_fp32 != 0; 16-byte aligned
 *   topk_idx   device int32 [T,K], e.g. from eqb_route_topk
 *   mask       device uint8 [T] (nullable)
 *   score      0 softmax, 1 normalised sigmoid (zeta must then be 0)
 *   alpha, zeta  any sign; alpha and 2 zeta finite in fp32
 *   grad_in    device fp32 [T,E], 16-byte aligned (nullable): a gradient with
 *              respect to z.  The path's grad_s is one with respect to s =
 *              sigma(z): it is multiplied by s (1 - s) before it is given here
 *   grad_out   device fp32 [T,E], or bf16 with grad_out_bf16 != 0 (rounded to
 *              nearest even: the operand of eqb_router_grad); 16-byte aligned
 *              (nullable: no gradient).  May be grad_in where both are fp32.
 *   grad_scale device fp32 [1] (nullable: 1): a loss scale
 *   counts     device int32 [M,E] (out, overwritten): f
 *   prob       device fp32 [M,E] (out, nullable): P
 *   loss       device fp32 [M,2] (out, nullable)
 *   workspace  device buffer of eqb_balance_loss_workspace_bytes(T, E, M)
 *              bytes, 256-byte aligned, needed unless prob, loss and mask are
 *              all NULL; nothing in it is kept between calls
 *   err_flag   EQB_ERR_NONFINITE for a NaN (softmax: or +inf) logit of a
 *              token that counts
 * Supported: E a multiple of 8 up to 1024, 1 <= K < E, K <= 31, T as above,
 * 1 <= M <= 2^20. */
size_t eqb_balance_loss_workspace_bytes(int64_t T, int32_t E, int32_t M);
eqb_status eqb_balance_loss(const void *z, int32_t z_fp32, const int32_t *topk_idx, int64_t T,
                            int32_t E, int32_t K, const int64_t *mb_offsets, int32_t M,
                            const uint8_t *mask, int32_t score, double alpha, double zeta,
                            const float *grad_in, void *grad_out, int32_t grad_out_bf16,
                            const float *grad_scale, int32_t *counts, float *prob, float *loss,
                            void *workspace, size_t workspace_bytes, int32_t *err_flag,
                            void *stream);

/* Gradients of the router projection z = x W_r^T (eqb_router_logits):
 *   dx[t, j] = sum_e dz[t, e] W_r[e, j]      (bf16)
 *   dW[e, j] = sum_t dz[t, e] x[t, j]        (fp32)
 * from bf16 inputs with fp32 accumulation on the tensor cores (tcgen05).  With
 * accumulate_dx or accumulate_dW the result is added to what the output holds
 * (in fp32, dx rounded once).  Either output may be NULL; then it is not
 * computed.  dW's tokens are summed 512 at a time on the tensor cores, the sums in
 * parts that depend on T, d, E, the SM count and which outputs are asked for, and
 * the parts in a fixed order: the same call gives the same bits.
 *   dz         device bf16 [T,E], 16-byte aligned, e.g. from eqb_balance_loss
 *   x          device bf16 [T,d], 16-byte aligned (not read without dW)
 *   W_r        device bf16 [E,d], 16-byte aligned (not read without dx)
 *   dx         device bf16 [T,d], 16-byte aligned, not overlapping x
 *   dW         device fp32 [E,d], 16-byte aligned
 *   workspace  device buffer of eqb_router_grad_workspace_bytes(T, d, E)
 *              bytes, 256-byte aligned (dW only; may be NULL where that is 0)
 *   err_flag   EQB_ERR_CUDA if a kernel's pipeline stalled and it gave up
 * Supported: d and E as in eqb_router_logits.  T = 0: dx is empty, dW is 0 (or
 * left as it is with accumulate_dW). */
size_t eqb_router_grad_workspace_bytes(int64_t T, int32_t d, int32_t E);
eqb_status eqb_router_grad(const eqb_bf16 *dz, const eqb_bf16 *x, const eqb_bf16 *W_r, int64_t T,
                           int32_t d, int32_t E, eqb_bf16 *dx, int32_t accumulate_dx, float *dW,
                           int32_t accumulate_dW, void *workspace, size_t workspace_bytes,
                           int32_t *err_flag, void *stream);

/* One AdamW step over many tensors (no counterpart in the paper: it is what
 * takes the gradients above back into the router and the experts).  For every
 * element, with g the gradient times grad_scale:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   p = (1 - lr weight_decay) p
 *       - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps).
 * The arithmetic is fp32, the factors are formed in fp64.  The update's quotient
 * is within 2 ulps, and so is its root, where a second moment below 2^-126 counts
 * as 0.  With 8 bits m, v, sqrt(v), scales and codes are rounded to nearest
 * operation by operation, without fused ones.  A bf16 parameter is rounded to
 * nearest once a step (an update below half its last place is lost: keep an fp32
 * parameter with a bf16 copy where that matters).
 * state_bits 32: exp_avg holds m and exp_avg_sq holds v, fp32 [n].
 * state_bits 8:  exp_avg holds m and exp_avg_sq holds sqrt(v) (whose range is
 *   half as many powers of two) in e4m3, one byte an element, each block of 256
 *   consecutive elements with an fp32 scale: the value is code * scale, scale =
 *   largest magnitude / 448, rounded to nearest even; a root that is not zero
 *   is not rounded to zero.  avg_scale, sq_scale: fp32 [ceil(n / 256)].  A block
 *   whose scale would be below 2^-126 is stored as zeros.
 *   Meant for beta2 up to 0.95: three places of mantissa cannot move a root by
 *   less than 3 to 6 % of itself against its block's scale.  Over thousands of
 *   steps of random gradients roots then scatter by 6 to 9 % around the true ones
 *   and stand up to 7 % above them; at 0.98 and 0.99 up to 60 and 35 % above, at
 *   0.999 they scatter by 15 to 24 %.  Decay alone moves the scale, not the codes: a
 *   root without gradients in a block that has some stays in step with that scale.
 * Zeroed states (and scales) are those of a first step.
 *   tensors    host array [count]; read before the call returns.  n >= 0; an
 *              entry with n = 0 or grad = NULL is left as it is.  Tensors must
 *              not overlap.  Any element alignment; arrays aligned to 16
 *              bytes are the fast path.
 *   lr, weight_decay  not negative; lr / (1 - beta1^step) and 1 - lr weight_decay
 *              finite in fp32
 *   eps        a normal number in fp32 (2^-126 <= eps < 2^128): where a gradient
 *              has been 0 so far it is all of the denominator
 *   grad_scale device fp32 [1] (nullable: 1): a clipping factor or the inverse
 *              of a loss scale, formed on the device
 *   err_flag   EQB_ERR_NONFINITE if a moment became non-finite (a gradient
 *              was, or its square is beyond fp32)
 * Up to 400 tensors share a launch. */
typedef struct eqb_adamw_tensor {
  void *param;      /* fp32 or bf16 [n], updated */
  const void *grad; /* fp32 or bf16 [n] */
  void *exp_avg;
  void *exp_avg_sq;
  float *avg_scale; /* state_bits 8 */
  float *sq_scale;
  eqb_bf16 *copy;   /* nullable, with an fp32 param: bf16 [n], the new param rounded */
  int64_t n;
  int32_t param_bf16;
  int32_t grad_bf16;
} eqb_adamw_tensor;
eqb_status eqb_adamw_step(const eqb_adamw_tensor *tensors, int32_t count, int32_t state_bits,
                          double lr, int64_t step, double beta1, double beta2, double eps,
                          double weight_decay, const float *grad_scale, int32_t *err_flag,
                          void *stream);

/* ---- The experts behind the router (no counterpart in the paper, which stops
 * at the lists: these take a list to the experts and back).
 *
 * Gate: experts and gate weights of every token, with experts in groups.  With
 * the choosing score c_e = fp32(z_{t,e}) + b_e (as in eqb_route_topk; z and b may
 * be -inf, which closes an expert):
 *   groups   with top_groups < groups, the experts are `groups` groups of
 *            E / groups neighbours; a group's score is its largest c, or with
 *            group_top2 the sum (fp32) of its two largest, where a second that is
 *            closed (or missing) counts nothing.  The top_groups best groups stay
 *            open (ties to the lower group);
 *   list     the K open experts of largest c > -inf, in descending order (ties to
 *            the lower expert); where fewer are open, the rest of the list is -1;
 *   weights  from the unbiased logits, s = sigmoid(z_t) or softmax(z_t) over all E
 *            experts: w_k = scale s_k, or with renorm scale s_k / (sum of the
 *            list's s).  An entry of -1 has weight 0.
 * Choice and ties are exact (fp32 sums and comparisons; -0 and +0 are equal); the
 * weights are fp32, renormalised without underflow however low the logits are.  Calls
 * of up to 4,096 tokens and calls of more divide and sum exponentials in other ways,
 * so the last places of a token's weights can differ between them; its list does not.
 *   z        device bf16 [T,E], or fp32 with z_fp32 != 0; 16-byte aligned
 *   b        device fp32 [E] (nullable: 0)
 *   mask     device uint8 [T] (nullable): a token whose byte is 0 gets -1 and
 *            0 throughout; its row of z is not looked at
 *   score    0 softmax, 1 sigmoid
 *   topk_idx device int32 [T,K] (out); weight device fp32 [T,K] (out, nullable)
 *   err_flag EQB_ERR_NONFINITE for a NaN or +inf c (or, with softmax, z) of a
 *            token that counts
 * Supported: E a multiple of 8 up to 1024, 1 <= K < E, K <= 31, groups <= 32 and
 * dividing E, 1 <= top_groups <= groups, K <= top_groups E / groups, scale
 * finite in fp32, T as above. */
eqb_status eqb_gate_topk(const void *z, int32_t z_fp32, const float *b, int64_t T, int32_t E, int32_t K,
                         int32_t groups, int32_t top_groups, int32_t group_top2, int32_t score,
                         int32_t renorm, double scale, const uint8_t *mask, int32_t *topk_idx,
                         float *weight, int32_t *err_flag, void *stream);

/* Gradient of eqb_gate_topk's weights with respect to z, the lists being
 * constants.  With g = dL/dw, and a_k = s_k / (sum of the list's s), gb = sum_k a_k g_k:
 *   sigmoid          d_k = scale g_k s_k (1 - s_k)
 *   sigmoid, renorm  d_k = scale a_k (1 - s_k) (g_k - gb)
 *   softmax, renorm  d_k = scale a_k (g_k - gb)
 *   softmax          d_j = scale p_j ([j in list] g_j - sum_k p_k g_k), every j
 * and 0 for experts outside the list in the first three.  grad_out = grad_in + d
 * (d without grad_in): dL/dz as eqb_balance_loss takes it in grad_in, or, in bf16,
 * eqb_router_grad in dz.  A list entry outside [0, E) has no part in anything, and a
 * token without any other has d = 0, whatever its row of z holds.  An expert that a
 * list names twice counts as two entries whose terms are added.  In the last kind a p
 * below 2^-126 counts as 0.
 *   z, z_fp32, score, renorm, scale  as in eqb_gate_topk
 *   topk_idx     device int32 [T,K]; grad_weight device fp32 [T,K]
 *   grad_in      device fp32 [T,E], 16-byte aligned (nullable); of the first three
 *                kinds only the lists' entries are touched where grad_out is grad_in
 *   grad_out     device fp32 [T,E], or bf16 with grad_out_bf16 != 0 (rounded once);
 *                16-byte aligned.  May be grad_in where both are fp32.
 * Supported: sizes as in eqb_gate_topk. */
eqb_status eqb_gate_grad(const void *z, int32_t z_fp32, const int32_t *topk_idx,
                         const float *grad_weight, int64_t T, int32_t E, int32_t K, int32_t score,
                         int32_t renorm, double scale, const float *grad_in, void *grad_out,
                         int32_t grad_out_bf16, void *stream);

/* The experts' rows: the entries of the lists (token t's k-th is entry t K + k)
 * that name an expert in [0, E), sorted by expert, within an expert in ascending
 * order.  Row r of the sorted order is what the calls below keep in row r of their
 * buffers of R = T K rows.
 *   offsets  device int32 [E+1] (out): expert e has rows offsets[e] .. offsets[e+1]-1
 *   blocks   device int32 [E+1] (out): expert e has blocks[e+1] - blocks[e] =
 *            ceil(rows / 128) blocks of 128 rows in eqb_quant_cols and eqb_expert_wgrad
 *   slot     device int32 [T,K] (out): the row of every entry, -1 where it has none
 *   entry    device int32 [T K] (out): the entry of every row, -1 behind the last
 *   workspace  device buffer of eqb_expert_rows_workspace_bytes(T, K, E) bytes,
 *            256-byte aligned (may be NULL where that is 0)
 * Supported: 1 <= E <= 1024, 1 <= K <= 1024, T K <= 2^31 - 2^24. */
size_t eqb_expert_rows_workspace_bytes(int64_t T, int32_t K, int32_t E);
eqb_status eqb_expert_rows(const int32_t *topk_idx, int64_t T, int32_t K, int32_t E, int32_t *offsets,
                           int32_t *blocks, int32_t *slot, int32_t *entry, void *workspace,
                           size_t workspace_bytes, void *stream);

/* Most blocks of 128 rows that R rows of E experts can have: what the buffers of
 * eqb_quant_cols are allocated for.  Host only; -1 for invalid arguments. */
int64_t eqb_expert_max_blocks(int64_t R, int32_t E);

/* Values in 8 bits (e4m3) with an fp32 scale for each block of 128 of them:
 *   scale = max |x| * fp32(1 / 448), 0 if below 2^-126,
 *   code  = e4m3_rne(clamp(x * fp32(1 / scale), -448, 448)), x's zero where scale is 0,
 * operation by operation in fp32 (x = code * scale to within half a step of
 * e4m3, 2^-4 of the value, or 2^-10 of the scale).  err_flag: EQB_ERR_NONFINITE
 * if a value that is read is not finite; its block's codes and scale are then
 * unspecified, and no other's.
 *
 * eqb_quant_rows: blocks of 128 neighbours in a row (the last of a row may be
 * shorter).  Without slot, row t of x becomes row t of q.  With slot [T,K], row t
 * becomes row slot[t,k] of q for every k whose slot lies in [0, T K); the others are
 * left out, and rows of q that no slot names are left as they are; a token without a
 * slot is not looked at.  Without slot all T rows are, and raise err_flag: of sorted rows
 * those behind the last expert's too, which the calls below do not write.  They hold finite
 * values (a buffer cleared when it is made), or are left out by a slot [R,1] of r, and -1
 * where entry[r] is.
 *   x      device bf16 [T,d], 16-byte aligned
 *   q      device e4m3 (one byte) [T,d], with slot [T K, d]; 16-byte aligned (out)
 *   scale  device fp32 [rows of q, ceil(d / 128)] (out)
 *   slot   device int32 [T,K] (nullable; then K is ignored), no row twice
 * Supported: d a multiple of 16 up to 2^20, T and T K <= 2^31 - 2^24. */
eqb_status eqb_quant_rows(const eqb_bf16 *x, int64_t T, int32_t d, const int32_t *slot, int32_t K,
                          uint8_t *q, float *scale, int32_t *err_flag, void *stream);

/* Blocks of 128 rows of an expert, for each column its own scale, turned: the
 * operands of eqb_expert_wgrad.  Row i of expert e's block b' (block number
 * b = blocks[e] + b') is the sorted row r = offsets[e] + 128 b' + i while that is
 * below offsets[e+1], and zeros after; its values are x[r], or with entry
 * x[entry[r] / K].
 *   x        device bf16 [R,c], with entry [T,c]; 16-byte aligned
 *   entry    device int32 [R] (nullable); an entry outside [0, T K) reads as zeros
 *   offsets, blocks  device int32 [E+1], from eqb_expert_rows
 *   q        device e4m3 [c, 128 P] (out), 16-byte aligned: q[j, 128 b + i]
 *   scale    device fp32 [P, c] (out)
 *   P        blocks allocated for: eqb_expert_max_blocks(R, E) is always enough.
 *            Blocks from blocks[E] on are left as they are; blocks from P on are not
 *            written.
 * Supported: c a multiple of 16 up to 2^20, E <= 1024, R, T <= 2^31 - 2^24,
 * P <= 2^24 - 2^17. */
eqb_status eqb_quant_cols(const eqb_bf16 *x, int64_t T, int32_t c, const int32_t *entry, int64_t R,
                          int32_t K, const int32_t *offsets, const int32_t *blocks, int32_t E,
                          int64_t P, uint8_t *q, float *scale, int32_t *err_flag, void *stream);

/* Blocks of 128 x 128 of each of E matrices, and, from the same read, of their
 * transposes (the same codes and scales, turned): the weights of
 * eqb_expert_matmul for the forward product and for the gradient of its input.
 *   w        device bf16 [E,n,d], or fp32 with w_fp32 != 0; 16-byte aligned
 *   q        device e4m3 [E,n,d]; scale device fp32 [E, ceil(n/128), ceil(d/128)]
 *   q_t      device e4m3 [E,d,n]; scale_t device fp32 [E, ceil(d/128), ceil(n/128)]
 *            (nullable, both together)
 * Supported: n and d multiples of 16 up to 2^20, 0 <= E <= 1024. */
eqb_status eqb_quant_blocks(const void *w, int32_t w_fp32, int32_t E, int32_t n, int32_t d, uint8_t *q,
                            float *scale, uint8_t *q_t, float *scale_t, int32_t *err_flag,
                            void *stream);

/* The experts' product in 8 bits.  For every row r of expert e:
 *   out[r, j] = sum over blocks B of 128 columns:
 *               scale[r, B] w_scale[e, j / 128, B] sum_{i in B} q[r, i] w[e, j, i].
 * The sum over a block is formed by the tensor cores (tcgen05, fp32), the sum
 * over the blocks in fp32 with one fused multiply-add each, in ascending order; out
 * is rounded once.  The same call gives the same bits.  With the transposed weights
 * of eqb_quant_blocks it is the gradient with respect to the input.
 *   q, scale    device e4m3 [R,d], fp32 [R, ceil(d/128)], from eqb_quant_rows; q
 *               16-byte aligned
 *   w, w_scale  device e4m3 [E,n,d], fp32 [E, ceil(n/128), ceil(d/128)]; w
 *               16-byte aligned
 *   offsets     device int32 [E+1]; read on the device, and kept within [0, R]
 *   out         device bf16 [R,n], or fp32 with out_fp32 != 0; 32-byte aligned.
 *               Rows from offsets[E] on are left as they are.
 *   err_flag    EQB_ERR_CUDA if a kernel's pipeline stalled and it gave up
 * Supported: n and d multiples of 16 up to 2^20, 1 <= E <= 1024, R <= 2^31 - 2^24. */
eqb_status eqb_expert_matmul(const uint8_t *q, const float *scale, const uint8_t *w,
                             const float *w_scale, const int32_t *offsets, int64_t R, int32_t n,
                             int32_t d, int32_t E, void *out, int32_t out_fp32, int32_t *err_flag,
                             void *stream);

/* The gradient of the experts' weights in 8 bits, from two buffers of
 * eqb_quant_cols over the same rows (a of the product's output gradient, b of its
 * input):
 *   dW[e, i, j] = sum over e's blocks B: a_scale[B, i] b_scale[B, j]
 *                 sum_{r in B} a[i, r] b[j, r]
 * with the sums of eqb_expert_matmul; with accumulate it is added to what dW
 * holds (in fp32).  An expert without blocks gets 0 (or is left as it is).
 *   a, a_scale  device e4m3 [n, 128 P], fp32 [P, n]; a 16-byte aligned
 *   b, b_scale  device e4m3 [d, 128 P], fp32 [P, d]; b 16-byte aligned, b_scale too
 *   blocks      device int32 [E+1]; read on the device, and kept within [0, P]
 *   dW          device fp32 [E,n,d], 32-byte aligned
 *   err_flag    as in eqb_expert_matmul
 * Supported: as in eqb_expert_matmul; P <= 2^24 - 2^17. */
eqb_status eqb_expert_wgrad(const uint8_t *a, const float *a_scale, const uint8_t *b,
                            const float *b_scale, const int32_t *blocks, int64_t P, int32_t n,
                            int32_t d, int32_t E, float *dW, int32_t accumulate, int32_t *err_flag,
                            void *stream);

/* The way back: out[t] = sum_k weight[t,k] rows[slot[t,k]] over the entries whose slot
 * lies in [0, R), in ascending k, fp32, rounded once; without weight the plain
 * sum (the gradient of the rows that eqb_quant_rows sent out).  Rows that no slot
 * names are not read.
 *   rows    device bf16 [R,n], 16-byte aligned
 *   slot    device int32 [T,K]; weight device fp32 [T,K] (nullable: 1)
 *   out     device bf16 [T,n], 16-byte aligned, not overlapping rows
 * Supported: n a multiple of 16 up to 2^20, 1 <= K <= 1024, T, R and T K
 * <= 2^31 - 2^24. */
eqb_status eqb_expert_combine(const eqb_bf16 *rows, const int32_t *slot, const float *weight, int64_t T,
                              int64_t R, int32_t n, int32_t K, eqb_bf16 *out, void *stream);

/* Its gradients from grad = dL/dout:
 *   grad_rows[slot[t,k]] = weight[t,k] grad[t]       (bf16, rounded once)
 *   grad_weight[t,k] = sum_j grad[t,j] rows[slot[t,k], j]   (fp32; 0 without a slot)
 * Either may be NULL.  Rows that no slot names are left as they are.
 *   grad       device bf16 [T,n], 16-byte aligned
 *   rows       as above (not read without grad_weight), weight too (nullable: 1)
 *   slot       no row twice
 *   grad_rows  device bf16 [R,n], 16-byte aligned; may be rows itself
 * Supported: as in eqb_expert_combine. */
eqb_status eqb_expert_combine_grad(const eqb_bf16 *grad, const eqb_bf16 *rows, const int32_t *slot,
                                   const float *weight, int64_t T, int64_t R, int32_t n, int32_t K,
                                   eqb_bf16 *grad_rows, float *grad_weight, void *stream);

/* Self-test of failure detection (no GPU fault involved): every wait in the
 * library's kernels is a bounded poll of a shared-memory mbarrier, and a
 * kernel whose pipeline stalls gives up, writes EQB_ERR_CUDA to its error
 * word and returns, leaving the context usable.  This call runs one block
 * that polls, `polls` times, a barrier that nothing completes, and reports
 * the stall the same way.  The paper has no counterpart.
 *   err_flag  device int32 (out): EQB_ERR_CUDA once the wait gives up
 *   polls     1 .. 2^24 */
eqb_status eqb_selftest_stalled_wait(int32_t *err_flag, int32_t polls, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EQB_H */
