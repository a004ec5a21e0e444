/*
 * libef21 -- the data-parallel hot path of EF21 (Richtarik, Sokolov, Fatkhullin,
 * arXiv 2106.05203) on one AMD MI355X (gfx950).  C ABI; no C++ or framework types cross it.
 *
 * The library solves the paper's problem  min_x f(x) = (1/n) sum_i f_i(x)  (eq. (1)) with
 * Algorithm 2 ("EF21, multiple nodes"), all n workers batched as rows on one GPU:
 *
 *     line 3   x   <- x - gamma * g
 *     line 5   c_i  = C(grad f_i(x) - g_i)          C = Top-k (Section 2.1)
 *     line 6   g_i <- g_i + c_i
 *     line 8   g   <- g + (1/n) sum_i c_i
 *
 * Conventions that hold for every call
 *   - Every array argument is a DEVICE pointer to memory the caller owns (for example the
 *     storage of a PyTorch tensor), row-major and contiguous.  Values are fp32, indices are
 *     int32, sizes are int64.  The library copies what it needs to keep (state); it only
 *     borrows problem data (see ef21_set_problem_*).
 *   - Work is enqueued on a HIP stream and the call returns without waiting for it.  The
 *     caller synchronises the stream before reading results on the host.
 *   - Every function except ef21_create and ef21_last_error returns an EF21_* status.  On
 *     failure nothing has been enqueued unless stated, and ef21_last_error() describes it.
 *   - NaN inputs are outside the contract: a NaN ranks above +inf in Top-k (its bit pattern
 *     is larger); nothing traps.
 *   - A handle is not thread safe; different handles may be used from different threads.
 */
#ifndef EF21_H
#define EF21_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ef21_ctx *ef21_handle;

enum {
    EF21_OK = 0,
    EF21_EINVAL = -1, /* bad argument (size, NULL pointer, gamma)                       */
    EF21_ENOMEM = -2, /* device or host allocation failed                                */
    EF21_EHIP = -3,   /* a HIP runtime call failed; text in ef21_last_error()            */
    EF21_ESTATE = -4  /* call not possible in the handle's state (e.g. no problem set)   */
};

/* flags of ef21_step (one order, optionally or-ed with EF21_PLUS or EF21_ONE_LAUNCH) */
enum {
    EF21_ORDER_GRAD_FIRST = 0u, /* lines 5, 6, 8 at the current x, then line 3 (default)      */
    EF21_ORDER_STEP_FIRST = 1u, /* line 3, then lines 5, 6, 8 at the new x (loop as printed)  */
    EF21_PLUS = 2u,             /* the loop body of Algorithm 3 (EF21+) instead of Algorithm 2 */
    EF21_CLASSIC_EF = 4u,       /* one round of Algorithm 4 (the original EF); no order, no EF21_PLUS */
    EF21_ONE_LAUNCH = 8u        /* the whole pass as one kernel where the problem qualifies (see ef21_step) */
};

/* Human-readable text of the calling thread's last failure ("" if none).  Library-owned. */
const char *ef21_last_error(void);

/*
 * Input line of Algorithm 2: n workers, dimension d, Top-k parameter k (1 <= k <= d), learning
 * rate gamma > 0 (finite).  Allocates, on the current HIP device, the state x [d], g [d],
 * g_i [n][d] (all zero) and the last messages (idx, val) [n][k].  Returns NULL on failure.
 * d must be below 2^31 (indices are int32) and n at most 65535 (a worker is a row of the launch grids).
 */
ef21_handle ef21_create(int32_t n, int64_t d, int64_t k, float gamma);

/* Waits for the handle's stream, then frees everything the handle owns.  NULL is allowed. */
int ef21_destroy(ef21_handle h);

/* Stream (a hipStream_t passed as void*) that later calls on this handle enqueue on.  The
 * stream is borrowed.  Default: the null stream. */
int ef21_set_stream(ef21_handle h, void *hip_stream);

/*
 * Top-k compressor of Section 2.1, batched over rows, stateless:  for each of the n rows of
 * `rows` [n][d] keep the k entries of largest absolute value.  Magnitudes are compared as
 * the fp32 bit pattern with the sign bit cleared, so +a ties with -a and +0 with -0; among
 * equal magnitudes the LOWER index is kept (the paper does not specify ties).
 *   out_idx [n][k]  kept positions of each row in ASCENDING order
 *   out_val [n][k]  the (signed) input values at those positions
 * Exactly k pairs are produced per row even if fewer than k entries are non-zero.
 * Enqueued on `hip_stream` (NULL = null stream).  For rows longer than a few 10^4 entries the
 * call uses a device workspace (about 8 d + 90 000 bytes per row) that the library keeps per device and
 * stream and grows on demand with hipMalloc (a growing call waits for that stream first).  Calls on
 * different streams use different workspaces and may overlap; calls on one stream run one after the other.
 * The workspaces are kept until the process ends (a device that has seen more than 16 streams frees all
 * of its workspaces after a device-wide wait and starts over).  ef21_topk_static never allocates.
 * EF21_EINVAL: n < 1, n > 65535 (a row is a row of the launch grids), d < 1, d >= 2^31, k < 1, k > d, NULL pointer.
 */
int ef21_topk(const float *rows, int32_t n, int64_t d, int64_t k, int32_t *out_idx, float *out_val,
              void *hip_stream);

/*
 * ef21_topk for callers that cannot allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, same results (the same kernels) as ef21_topk, but the workspace
 * of the long-row path is a 64 MiB array that is part of the library's device image (each GPU the library runs on
 * holds it until the process ends), so the call allocates nothing, frees nothing and synchronises nothing: it
 * enqueues kernels on `hip_stream` and returns.  Rows of 16384 entries or more that are not selected by one
 * workgroup per row (d > 61440 or k > 1024) need about 8 d + 90 000 bytes of workspace per row; a call whose
 * n rows need more than the 64 MiB (for example more than eight rows of 10^6 entries) is rejected with EF21_EINVAL
 * and a message that gives both sizes -- use ef21_topk for those.  Shorter rows need no workspace and have no limit.
 * Every call on a GPU shares that GPU's array: calls that overlap on one GPU (two streams, two threads) race and
 * give wrong results; calls that follow one another on a stream, of any shapes, are fine (each call clears the
 * part of the array that must start at zero with a fill kernel of its own, so it may also be captured into a graph).
 * Errors otherwise as ef21_topk.
 */
int ef21_topk_static(const float *rows, int32_t n, int64_t d, int64_t k, int32_t *out_idx, float *out_val,
                     void *hip_stream);

/*
 * Attach the objective of Section 5, eq. (9): logistic loss with the non-convex regulariser,
 *   f_i(x) = (1/m) sum_l log(1 + exp(-y_il a_il^T x)) + lambda sum_j x_j^2 / (1 + x_j^2),
 * each worker holding m rows (each f_i carries the full regulariser, so (1/n) sum_i f_i is
 * eq. (9) for an even split of the data).
 *   dense:  A [n][m][d] fp32, y [n][m] fp32 in {-1, +1}
 *   csr:    one CSR over all n*m rows, worker i owning rows i*m .. (i+1)*m-1:
 *           rowptr [n*m+1] int64, col [nnz] int32 in [0, d), val [nnz] fp32, y [n][m]
 * The arrays are BORROWED: they must stay valid and unchanged while the handle uses them.
 * Allocates a gradient buffer [n][d] and scratch on first use.  The csr call also reads the matrix
 * once (it waits for the stream): if every row's columns are strictly ascending and inside [0, d),
 * and no worker holds 2^31 - 2^16 entries or more, it builds what the fast two-pass gradient kernels
 * need -- a small per-row index of column ranges and two re-ordered copies of the matrix with 16-bit
 * indices (about 12 bytes per entry plus 4 n (d + 1) + 4 (n m + n) ceil(d / 12288) bytes of device
 * memory in all, owned by the handle).  Otherwise a slower kernel based on global floating-point
 * atomics is used, in which columns outside [0, d) are skipped.
 */
int ef21_set_problem_dense(ef21_handle h, const float *A, const float *y, int64_t m, float lambda);
int ef21_set_problem_csr(ef21_handle h, const int64_t *rowptr, const int32_t *col, const float *val,
                         const float *y, int64_t m, float lambda);

/*
 * The per-row loss of the attached problem (default EF21_LOSS_LOGISTIC).  With EF21_LOSS_LEAST_SQUARES the
 * objective is the one of Section 5.2,
 *   f_i(x) = (1/m) sum_l (a_il^T x - y_il)^2  (+ the regulariser of eq. (9) times lambda; pass lambda = 0 for
 *   the paper's function), y holding the targets b_il,
 * whose gradient is (2/m) sum_l (a_il^T x - y_il) a_il: the same kernels with another derivative per row.
 * Takes effect from the next gradient.  EF21_EINVAL: unknown value.
 */
enum { EF21_LOSS_LOGISTIC = 0, EF21_LOSS_LEAST_SQUARES = 1 };
int ef21_set_loss(ef21_handle h, int loss);

/*
 * Stochastic gradients (Algorithm 5, the extension of Algorithm 2 in the appendix): from the next gradient
 * on, worker i's gradient is replaced by the minibatch estimator
 *   ghat_i = (1/tau) sum over l in rows[i][0..tau) of the gradient of row l's loss  +  the regulariser's,
 * in ef21_local_grad and in every variant of ef21_step.  rows: device, int32 [n][tau], row numbers inside
 * the worker's m rows, drawn by the caller (the library draws no random numbers); borrowed and read at
 * every gradient, so the caller redraws a batch by rewriting the buffer (stream-ordered) or by another call.
 * A row listed twice counts twice; an entry outside [0, m) contributes nothing and is never dereferenced
 * (the division stays by tau).  tau == 0 (rows ignored): back to the full gradient.  Attaching a problem
 * resets it.  Dense rows run the ordinary kernels over the listed rows (bitwise reproducible); CSR rows take
 * one wavefront per listed row and global fp32 atomics (reproducible to rounding), work proportional to
 * the batch.  EF21_ESTATE without a problem; EF21_EINVAL: tau outside [0, m], or rows NULL with tau > 0.
 */
int ef21_set_minibatch(ef21_handle h, const int32_t *rows, int64_t tau);

/*
 * The largest stepsize Theorem 1 allows for the attached problem (Section 3.4, the bound on gamma in the theorem),
 *   gamma = 1 / (L + Ltilde sqrt(beta / theta)),   sqrt(beta / theta) = (1 + sqrt(1 - alpha)) / alpha - 1,
 * alpha = k / d for Top-k, Ltilde the quadratic mean of the workers' smoothness constants
 *   L_i = c lambda_max((1/m) A_i^T A_i) + 2 lambda
 * (c = 1/4 for the logistic loss, 2 for least squares: the largest curvature of the per-row loss; 2 is the
 * largest curvature of t^2 / (1 + t^2)), and L = c lambda_max((1/(n m)) sum_i A_i^T A_i) + 2 lambda for f itself.
 * The eigenvalues are the estimates that `iterations` steps of the power iteration give on the GPU, started from a fixed
 * positive vector: the estimate |M v| for the unit vector v of the last step approaches lambda_max from below, so few
 * iterations give a stepsize that is
 * too large by the same factor: 100 to 300 steps bring problems without a dominant direction within about one
 * per cent.  gamma, L, L_i [n]: host memory, each may be NULL.  Uses the handle's loss, lambda and k, and all
 * rows whatever ef21_set_minibatch says; the handle's stepsize is not changed.  Returns after the stream has drained.
 * A dense problem with d <= 1024 columns is iterated on the workers' Gram matrices where that is the faster way (it is from
 * some ten iterations on, usually); many iterations are then not run one by one, but their estimate is taken, to fp64 rounding,
 * from powers of the matrices by repeated squaring, or (48 to 2822 iterations) from
 * ceil(4.8 sqrt(iterations)) + 1 steps of the Lanczos recurrence on the same start vector, whichever is estimated to be faster.
 * A call that needs more than the handle has allocates a workspace of
 * 4 (n + 1) d'^2 + 4 n c d' (d' + 32) + 8 (n + 1) (5 d' + 512) bytes (d' = d rounded up to 32, c pieces of a worker's rows, one
 * or as many as make a thousand tiles in all; by squaring 24 (n + 1) d'^2, or 16 (n + 1) d'^2 + 4 n c d' (d' + 32) where that is more,
 * and 16 (n + 1) (d' + 96)) and some ten thousand for alignment, never more than 1 GiB, which the handle
 * keeps until ef21_destroy (while a larger one is being allocated, what is there stays if it would do without squaring).
 * Where there is no memory for squaring a call goes without it; where there is none for the matrices, and for all other problems, it iterates with the
 * problem itself, a step two passes
 * of the gradient kernels over it: the first one
 * on a handle allocates (n + 2) d floats that the handle keeps, and every one overwrites the handle's gradient buffer.
 * EF21_ESTATE without a problem; EF21_EINVAL: iterations outside [1, 10^6]; EF21_ENOMEM.
 */
int ef21_theory_stepsize(ef21_handle h, int32_t iterations, double *gamma, double *L, double *L_i);

/*
 * State of Algorithm 2.  set: copies x [d] and g_i [n][d] into the handle (either may be NULL
 * = keep); g [d] NULL means "recompute g = (1/n) sum_i g_i" (the algorithm's input line).
 * get: copies the handle's state out; any pointer may be NULL.
 */
int ef21_set_state(ef21_handle h, const float *x, const float *g_i, const float *g);
int ef21_get_state(ef21_handle h, float *x, float *g_i, float *g);

/* The messages c_i of the last ef21_step as (idx, val) [n][k], layout as in ef21_topk. */
int ef21_get_messages(ef21_handle h, int32_t *idx, float *val);

/*
 * grad f_i(x) for all workers (derivative of eq. (9)):
 *   (1/m) sum_l  -y_il / (1 + exp(y_il a_il^T x)) a_il  +  2 lambda x_j / (1 + x_j^2)^2
 * at `x` [d] (NULL = the handle's x), written to out_grad [n][d].  EF21_ESTATE without a
 * problem.  fp32 arithmetic; sums over rows are taken in a fixed order (bitwise reproducible),
 * except in the atomics-based kernel for CSR rows with unsorted columns (reproducible to rounding).
 */
int ef21_local_grad(ef21_handle h, const float *x, float *out_grad);

/*
 * One pass of the loop body of Algorithm 2 for all workers.
 *   grads [n][d]: the vectors used in place of grad f_i(x) in line 5 (supplied gradients,
 *   e.g. the stochastic estimators of Algorithm 5), or NULL to compute grad f_i at the
 *   handle's x from the attached problem (EF21_ESTATE if none).
 *   flags: EF21_ORDER_GRAD_FIRST or EF21_ORDER_STEP_FIRST.  With supplied gradients and
 *   STEP_FIRST the caller must have evaluated them at x - gamma*g.
 * The difference in line 5 is one fp32 subtraction; line 6 is one fp32 addition per kept
 * entry; line 8 adds the messages per coordinate in fp32 and applies
 * g + sum * (1/n) as one fused multiply-add; line 3 is one fused multiply-add per coordinate.
 * The sum of line 8 takes the workers in order where n < 16, and where d <= 1024, n k <= 2048 and n ceil(k / 64) <= 512.
 * In all other calls it is ((r0 + r1) + r2) + r3 of the sums r0 .. r3, each in worker order, over four runs of
 * ceil(n / 4) consecutive workers (the last may hold fewer): the order depends on n, d and k alone.
 * With supplied gradients every result (messages, g_i, g, x) is bitwise reproducible.
 * With EF21_ONE_LAUNCH in flags, a small dense problem (grads NULL, d <= 1024, n * k <= 2048,
 * n * m * d <= 2^24, no minibatch, no EF21_PLUS) runs the whole pass as ONE kernel: the same arithmetic in the
 * same order as without the flag, so the results are the same bits.  It saves one launch (two where a worker's rows are
 * too many for one workgroup) and pays for it in device-scope fences: measured within five per cent of the
 * default for a few workers with a few hundred rows of 100 columns (calls back to back: n = 4, m = 250, d = 100 8.7 us against
 * 8.6, m = 500 10.2 against 10.4) and slower for larger problems and more workers (n = 20, m = 1628,
 * d = 123: 20.3 against 13.3), hence not the default.  Where the problem does not qualify the flag changes nothing.
 * EF21_EINVAL: unknown flag bits, or EF21_CLASSIC_EF together with an order or EF21_PLUS.
 */
int ef21_step(ef21_handle h, const float *grads, uint32_t flags);

/*
 * With EF21_PLUS in flags, ef21_step runs the loop body of Algorithm 3 (EF21+, Section 3.5) on the same
 * state: with s = grad f_i(x) (or the supplied row) every worker forms b = C(s) (line 5) and
 * m = g_i + C(s - g_i) (line 6), C = Top-k as in ef21_topk; the distortions B = ||b - s||^2 and
 * M = ||m - s||^2 (line 7) are computed in fp64 as ||s||^2 and ||s - g_i||^2 minus the sums of the kept
 * squares, every sum in a fixed order; g_i <- m if M <= B, else b (line 8); g <- (1/n) sum_i g_i, the
 * rows added in worker order in fp64 and the mean rounded once (line 10).  ef21_get_messages then returns, per worker, the k pairs
 * of the compressor it chose.  The first such call on a handle allocates (and waits for the stream): 16 n k bytes for
 * the two selections, and for rows of 16384 entries or more with k > 1 a second Top-k workspace (about 8 d + 90 000 bytes
 * per row, as the first, which a handle has from the start if d > 61440 or k > 1024 and else gets here) and, where there is
 * room for it, 4 n d bytes more (without them the step is slower).
 *
 * ef21_get_choices copies out what the last EF21_PLUS step decided: branch [n] int32 (1 = the plain
 * compressor b was chosen, 0 = the Markov compressor m) and distortions [n][2] fp64 (B_i, M_i); either
 * pointer may be NULL.  EF21_ESTATE before the first EF21_PLUS step.
 */
int ef21_get_choices(ef21_handle h, int32_t *branch, double *distortions);

/*
 * With flags == EF21_CLASSIC_EF, ef21_step runs one round of Algorithm 4 (EF, the original error feedback
 * that Section 4 compares EF21 with) on the same handle, the workers' errors e_i taking the place of g_i in
 * ef21_set_state / ef21_get_state (start from e_i = 0): at the handle's x, with s = grad f_i(x) or the
 * supplied row,  p_i = e_i + gamma s  (one fused multiply-add per entry, written over e_i),
 * w_i = C(p_i)  (Top-k as in ef21_topk; returned by ef21_get_messages),  e_i = p_i - w_i  (zero at the kept
 * positions),  x <- x - (1/n) sum_i w_i  (the sum per coordinate in fp32, in the order of line 8 of ef21_step).  Started from
 * e_i = 0 this produces the iterates x^0, x^1, ... of Algorithm 4.  The g of ef21_get_state holds
 * (1/n) sum_i w_i of the last round.  Do not mix rounds of different algorithms on one state.
 */

/*
 * Per-kernel timing, for measurement only (not part of the paper's method).  While enabled,
 * ef21_step and ef21_local_grad record one HIP event on the handle's stream after each kernel
 * they launch; the time between consecutive events is charged to the class of the later kernel.
 * ef21_set_timing and ef21_get_timing wait for the stream.  ms[EF21_K_COUNT] receives the
 * accumulated milliseconds per class and launches[EF21_K_COUNT] the number of intervals (either
 * may be NULL); reset != 0 clears the sums.  Classes, in order (names from ef21_kernel_name):
 * grad_main, grad_aux, topk_row, topk_collect, topk_select, topk_refine (no kernel; the number stays), topk_count, topk_emit,
 * model_step, plus (what is particular to Algorithm 3), small_step (the one-launch iteration).
 */
enum { EF21_K_COUNT = 11 };
int ef21_set_timing(ef21_handle h, int enabled);
int ef21_get_timing(ef21_handle h, double *ms, int64_t *launches, int reset);
const char *ef21_kernel_name(int kernel_class);

/*
 * Plain streaming kernels, for measurement only (not part of the paper's method): what this GPU's HBM
 * delivers to the simplest possible kernel, to set beside the vendor's peak.  Both take DEVICE pointers to
 * 16-byte aligned buffers of `bytes` bytes (a multiple of 16) and enqueue one kernel on `hip_stream`.
 *   ef21_hbm_read   reads `src` once with the same non-temporal loads the library's kernels use and
 *                   writes one float to sink[0] (sink may alias nothing else)
 *   ef21_hbm_copy   dst <- src
 * EF21_EINVAL: NULL pointer, misaligned pointer, bytes < 16 or not a multiple of 16.
 */
int ef21_hbm_read(const void *src, int64_t bytes, float *sink, void *hip_stream);
int ef21_hbm_copy(void *dst, const void *src, int64_t bytes, void *hip_stream);

/*
 * ---- The two ends of a language model ----
 * The lookup of an embedding table and the losses on a model's logits, with the gradients that ef21_step takes.  Stateless:
 * every call works on the arrays and the stream it is given, allocates and synchronises nothing (so it may be captured into a
 * HIP graph), and where it needs scratch memory the caller passes a workspace, of which a second call of the same function tells the size.
 * Tables, activations, logits and their gradients are fp32, bf16 or fp16 (EF21_F32, EF21_BF16, EF21_F16); arithmetic is fp32 and
 * results are rounded once, to nearest.  Tokens and labels are int32 or int64 (EF21_I32, EF21_I64).  Two-dimensional arrays
 * have contiguous rows `stride` entries apart, of any alignment that their type has.  Zero rows or tokens are allowed (then
 * the arrays that would be empty may be NULL).  Every result is bitwise reproducible.
 * EF21_EINVAL: a size or stride out of range, an unknown type, a NULL or misaligned pointer, a workspace that is too small.
 */
enum { EF21_F32 = 0, EF21_BF16 = 1, EF21_F16 = 2 };
enum { EF21_I32 = 0, EF21_I64 = 1 };

/*
 * Embedding lookup: out[t] = scale * table[tokens[t]] for `count` tokens, table [vocab][width], out [count][width].  A token
 * outside [0, vocab) is never dereferenced and gives a row of zeros.  out must not overlap the table.
 */
int ef21_embed(const void *table, int table_type, int64_t vocab, int64_t width, int64_t table_stride, const void *tokens,
               int token_type, int64_t count, float scale, void *out, int out_type, int64_t out_stride, void *hip_stream);

/*
 * Its gradient for n workers at once, each with `count` tokens: for worker i
 *   G_i[v] = scale * sum over t with tokens[i][t] = v of grad_out[i][t]          v = 0 .. vocab - 1
 * grad_out: [n][count] rows of `width` entries, grad_stride apart;  tokens [n][count];  G_i: fp32 [vocab][width], contiguous, at
 * table_grad + i * worker_stride -- with worker_stride = d a block of the rows [n][d] that ef21_step takes.  accumulate != 0
 * adds to what is there (a table shared with the output layer) and leaves rows without a token untouched; 0 writes every row.
 * Tokens outside [0, vocab) contribute nothing.  The positions are sorted by token and a token's rows are added in an order
 * that n, count, width and the tokens fix: the same call gives the same bits, another number of workers may round differently.
 * n in [1, 65535], count and vocab below 2^31.
 * workspace: 256-byte aligned device memory of at least the bytes that ef21_embed_grad_workspace says.
 */
int ef21_embed_grad_workspace(int32_t n, int64_t count, int64_t vocab, int64_t width, int64_t *bytes);
int ef21_embed_grad(const void *grad_out, int type, int64_t grad_stride, const void *tokens, int token_type, int32_t n,
                    int64_t count, int64_t vocab, int64_t width, float scale, float *table_grad, int64_t worker_stride,
                    int accumulate, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * Log-probabilities of the labels under the softmax of each row of logits [rows][vocab]:
 *   lse[r] = log sum_v exp(x_v),   logp[r] = x_label - lse[r]
 * A row whose label is outside [0, vocab) (a prompt's token, padding) is ignored here and in the calls below: it is not read,
 * its logp and lse are 0, its gradient is a row of zeros.  Entries of -inf have probability zero; a row with nothing above
 * -inf has lse = logp = -inf and a gradient of zeros.  A NaN or +inf in a row with a label makes that row's results NaN.
 */
int ef21_token_logps(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                     int label_type, float *logp, float *lse, void *hip_stream);

/*
 * The gradient of the logits from that of the log-probabilities, grad_logp [rows] (read where there is a label):
 *   grad_logits[r][v] = grad_logp[r] * ([v = label] - exp(x_v - lse[r]))
 * lse as ef21_token_logps gave it.  grad_logits has the logits' type; it may be the logits themselves (same stride) and must
 * otherwise not overlap them, here and in the calls below.  A row whose grad_logp (or, below, whose loss's derivative in logp) is
 * infinite has infinities where the factor in parentheses is not zero and zero where it is.
 */
int ef21_token_logps_grad(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                          int label_type, const float *lse, const float *grad_logp, void *grad_logits, int64_t grad_stride,
                          void *hip_stream);

/*
 * Preference loss of `pairs` pairs of sequences, the logistic or least squares loss of the difference of their log ratios to
 * a reference model.  Sequence s is the rows seq_start[s] .. seq_start[s + 1] - 1 of the logits (int64 [2 pairs + 1], device, not
 * decreasing, within [0, rows]; a sequence may be empty, and rows in none have a gradient of zeros); pair p prefers sequence
 * 2p to 2p + 1.  With S(s) the sum (mean != 0: the mean) over its labelled rows of logp - ref_logp and D = S(2p) - S(2p + 1):
 *   EF21_LOSS_LOGISTIC       out_loss[p] = -(1 - smoothing) log sigma(beta D) - smoothing log sigma(-beta D)
 *   EF21_LOSS_LEAST_SQUARES  out_loss[p] = (D - 1 / (2 beta))^2                      (smoothing plays no part)
 * ref_logp [rows]: the reference's log-probabilities per token (ef21_token_logps on its logits), read where there is a label;
 * per token, since of the sums over long sequences fp32 keeps too little.  logp [rows]: out.  grad_logits: the gradient of
 * sum_p pair_weight[p] out_loss[p], or NULL for the loss alone; pair_weight [pairs] or NULL for 1 / pairs.
 * EF21_EINVAL also: pairs < 1, beta not finite and > 0, smoothing outside [0, 1).
 * workspace: 256-byte aligned device memory of at least the bytes that ef21_preference_loss_workspace says.
 */
int ef21_preference_loss_workspace(int64_t rows, int32_t pairs, int64_t *bytes);
int ef21_preference_loss(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                         int label_type, const int64_t *seq_start, int32_t pairs, const float *ref_logp, float beta,
                         float smoothing, int loss, int mean, const float *pair_weight, float *out_loss, float *logp,
                         void *grad_logits, int64_t grad_stride, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * Clipped policy loss with a KL term, per token: with q = exp(logp - old_logp), A = advantages, o = ref_logp - logp
 *   token_loss[r] = -min(q A, clip(q, 1 - clip_low, 1 + clip_high) A) + kl (exp(o) - 1 - o)
 *   out_loss[0]   = sum_r weight[r] token_loss[r]
 * old_logp, advantages, ref_logp, weight: fp32 [rows], read where there is a label.  ref_logp NULL: no KL term (kl must be 0);
 * weight NULL: 1 / rows.  grad_logits: the gradient of out_loss, or NULL for the loss alone; where the two sides of the
 * minimum are equal it is that of q A.  token_loss and logp: fp32 [rows], out.  With a KL term a label of probability zero
 * (logp = -inf, ref_logp finite) has a token_loss and so an out_loss of +inf, and an infinite derivative in logp.
 * EF21_EINVAL also: clip_low outside [0, 1], clip_high or kl negative or not finite.
 * workspace: 256-byte aligned device memory of at least the bytes that ef21_policy_loss_workspace says.
 */
int ef21_policy_loss_workspace(int64_t rows, int64_t *bytes);
int ef21_policy_loss(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                     int label_type, const float *old_logp, const float *advantages, const float *ref_logp,
                     const float *weight, float clip_low, float clip_high, float kl, float *out_loss, float *token_loss,
                     float *logp, void *grad_logits, int64_t grad_stride, void *workspace, int64_t workspace_bytes,
                     void *hip_stream);

/*
 * What a model says about each row of logits: log-probabilities of given tokens, the entropy and the k most likely tokens,
 *   lse[r] = log sum_v exp(x_v),  logp[r] = x_label - lse[r],  entropy[r] = -sum_v p_v log p_v with p_v = exp(x_v - lse[r])
 *   top_tokens, top_logp [rows][k]: the k tokens of largest x_v in descending order, ties to the lower token, and x_v - lse[r]
 * labels [rows]: rows whose label is outside [0, vocab) are ignored: they are not read, their logp, lse, entropy and top_logp are 0 and their
 * top_tokens -1.  labels NULL (with any label_type): there are none, every row is taken, and logp must be NULL too.
 * k in [0, 64] and at most vocab; with k = 0 top_tokens and top_logp may be NULL.  sums: fp32 [rows][2] for ef21_token_stats_grad, whose
 * contents are that call's business, or NULL.
 * Entries of -inf have probability zero and take no part in the entropy; they are alternatives too, behind all others, of log-probability -inf.
 * A row with nothing above -inf has lse = logp = -inf and entropy 0.  A NaN or +inf in a row that is read makes its results NaN and its
 * top_tokens -1.  A row's results depend on its entries and its alignment alone, not on how many rows there are.
 * workspace: 256-byte aligned device memory of at least the bytes that ef21_token_stats_workspace says (0 where there are many rows).
 * EF21_EINVAL also: k out of range, logp without labels or labels without logp.
 */
int ef21_token_stats_workspace(int type, int64_t rows, int64_t vocab, int32_t k, int64_t *bytes);
int ef21_token_stats(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                     int label_type, int32_t k, float *logp, float *lse, float *entropy, int32_t *top_tokens, float *top_logp,
                     float *sums, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * The gradient of the logits from those of the log-probabilities and of the entropies,
 *   grad_logits[r][v] = grad_logp[r] * ([v = label] - p_v) - grad_entropy[r] * p_v * (log p_v + entropy[r])
 * sums and entropy as ef21_token_stats gave them for these logits and labels.  grad_logp or grad_entropy may be NULL (zero); without labels
 * grad_logp must be.  Both are finite and are read in the rows that count.  accumulate != 0 adds to what is in grad_logits (the gradient of
 * another loss; rounded once more, and rows that are ignored stay as they are) and then grad_logits must not be the logits; else it may be.
 * Ignored rows and rows with nothing above -inf have a gradient of zero, and so have entries of probability zero but for the label's: as the
 * formula says, that has grad_logp[r], also where it is -inf itself.
 */
int ef21_token_stats_grad(const void *logits, int type, int64_t rows, int64_t vocab, int64_t stride, const void *labels,
                          int label_type, const float *sums, const float *entropy, const float *grad_logp,
                          const float *grad_entropy, void *grad_logits, int64_t grad_stride, int accumulate, void *hip_stream);

/*
 * ---- The step of a model's parameters ----
 * Line 3 of Algorithm 2, x <- x - gamma g, is one way to use the estimate g of the gradient; these calls are another, over many tensors at
 * once: g may be parts of the vector that ef21_get_state gives, or any gradients.  Stateless, as the section above: nothing is allocated or
 * synchronised, the calls may be captured, results are bitwise reproducible.  Arrays of `tensor_count` entries are HOST memory and are
 * read before the call returns; what their pointers name is device memory, contiguous, aligned as its type is.  Tensors of count 0
 * are allowed (their pointers may be NULL), and so is tensor_count = 0.
 */

/*
 * The norm of many gradients together, and the factor that clips it:
 *   norm[0] = scale * sqrt(sum over all tensors and entries of g^2),   factor[0] = scale * min(1, max_norm / norm[0])
 * scale > 0: what the gradients still have to be multiplied by (1 / loss scale).  max_norm > 0; INFINITY clips nothing.  Squares and their
 * sum are fp64, in an order that the counts and types fix.  Where norm[0] is not finite factor[0] is NaN, which ef21_adamw takes for a step
 * to be skipped.
 * workspace: 256-byte aligned device memory of at least the bytes that ef21_grad_norm_workspace says.  It may hold anything; a call that follows
 * another with the same workspace finds its counter of workgroups ready.  Calls that share it must follow each other.
 */
int ef21_grad_norm_workspace(int32_t tensor_count, int64_t *bytes);
int ef21_grad_norm(const void *const *grads, const int32_t *types, const int64_t *counts, int32_t tensor_count, float scale,
                   float max_norm, float *norm, float *factor, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * AdamW (decoupled weight decay) over many tensors.  For every entry, with f = grad_scale[0] (1 if NULL) and t = step:
 *   g' = f g,   m <- beta1 m + (1 - beta1) g',   v <- beta2 v + (1 - beta2) g'^2
 *   p <- p - lr * (weight_decay * p + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps))
 * in fp32; with 8-bit states each product and sum of m and v is rounded by itself, so that the codes do not depend on how it is evaluated.
 * Where f is not finite nothing is changed.  An infinite or NaN gradient otherwise passes into m, v and p, of its entry alone with 32-bit
 * states; of 8-bit ones an infinity makes its block NaN (from the next step on where it is v's alone: that of a finite g' from 1.9e19 on, whose square
 * is rounded by itself).  A v that is NaN makes its p NaN, and so does a quotient beyond fp32.
 *   states: m, v fp32 (m_scale and v_scale NULL), or 8 bits: entry i of m stands for m_scale[i / 256] times the value of byte i as an OCP
 *           e4m3 number, and sqrt(v) for v_scale[i / 256] times that of v's byte; the scales, ceil(count / 256) of each, are the block's
 *           largest value / 448, 2^-126 at the least.  The update uses m and v before they are rounded to 8 bits.  A sqrt(v) above zero is
 *           never rounded to zero.
 *   copy:   NULL, or with fp32 parameters bf16 or fp16 [count] (copy_type): receives the new parameters, rounded to nearest
 *   stochastic != 0: what is kept in fewer than 32 bits (8-bit states, bf16 or fp16 parameters) is rounded up or down at random, with
 *           probabilities that make it right on average; a moving average that moves by 1 - beta of itself a step, or a parameter by
 *           less than half of its last bit, would stay where it is if it were rounded to nearest.  The choice follows from seed, step, the
 *           tensor's number in the call and the entry's, so that the same call gives the same bits.
 * lr_device, step_device: NULL, or fp32 [1] and int64 [1] that are read on the device in the place of lr and step (a captured call whose
 * values change; a step below 1 counts as 1).
 * The written arrays (param, m, v, their scales, copy) must not overlap one another or the gradients; no tensor may be listed twice.
 * EF21_EINVAL: a count < 0 or > 2^33, an unknown type, a NULL or misaligned pointer, one scale without the other, lr or weight_decay not finite,
 * beta1 or beta2 outside [0, 1), eps not finite and at least 2^-126, step < 1.
 */
typedef struct ef21_adamw_tensor {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    void *copy;
    int64_t count;
    int32_t param_type, grad_type, copy_type;
    float weight_decay;
} ef21_adamw_tensor;

typedef struct ef21_adamw_options {
    double lr, beta1, beta2, eps;    /* 1 - 0.999 in fp32 is 1e-5 of itself off */
    int64_t step;
    const float *lr_device;
    const int64_t *step_device;
    const float *grad_scale;
    uint64_t seed;
    int32_t stochastic;
} ef21_adamw_options;

int ef21_adamw(const ef21_adamw_tensor *tensors, int32_t tensor_count, const ef21_adamw_options *options, void *hip_stream);

/*
 * The same with the step's number counted on the device, where the host does not know which steps are skipped: counter is 16 bytes of device
 * memory, 8-byte aligned, that begin with the int64 number of the last step taken (0 at first, below 0 counts as 0; the caller may set it between
 * calls) and are otherwise the call's own.  Where f is finite the number goes up by one and is the step's; where it is not, it stays.  A captured
 * call counts at every replay.  options->step is not read, and options->step_device must be NULL.
 */
int ef21_adamw_counted(const ef21_adamw_tensor *tensors, int32_t tensor_count, const ef21_adamw_options *options, void *counter, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EF21_H */
