/*
 * kvdro.h -- C ABI of the GB300 Wasserstein-DRO KV-reservation grid evaluator.
 *
 * The library evaluates, on one GPU, the worst-case expected reservation cost
 * of the paper "Robust KV Cache Management for LLM Serving under Output Token
 * Length Uncertainty" over a grid of
 *     regimes m (a (c_p, c_w) pair) x classes k x reservations r x multipliers lam x radii eps
 * and reduces it to a per-(regime, radius, class) reservation.  For class k with
 * samples x_1..x_N (output lengths in tokens), support [0, L_k] and input
 * length L_in_k, with eta = r - L_in_k:
 *
 *   Q(eta, xi)   = c_p (xi - eta)^+ + c_w (eta - xi)^+                 (Sec. 2.3; App. A Step 1)
 *   phi_n        = max{ Q(eta,0) - lam x_n, Q(eta,x_n), Q(eta,L) - lam (L - x_n) }
 *                                                                       (App. A Step 4)
 *   S(eta, lam)  = (1/N) sum_n phi_n                                   (App. A Step 3)
 *   cost(eta,eps)= min_j ( lam_j eps + S(eta, lam_j) )                 (App. A eq. app_kantorovich,
 *                                                                        gamma restricted to the lam grid)
 *   r*           = argmin_r cost                                        (Sec. 2.4, eq. dro_obj, r block)
 *   quantiles    = lower empirical quantiles x_(max(1, ceil(q N)))     (Prop. "Critical Fractile
 *                                                                        Structure", eq. critical_fractile)
 *
 * Conventions shared by every entry point
 *   - Every function returns a kvdro_status.  Nothing is thrown or aborted across the ABI.
 *   - Argument errors are found on the host before any launch (KVDRO_EINVAL) and leave the
 *     context unchanged; kvdro_last_error() then describes the error.
 *   - Work is enqueued on `stream` (a cudaStream_t; NULL = the legacy default stream).
 *     Asynchronous CUDA errors surface at the next call or at kvdro_sync() (KVDRO_ECUDA).
 *   - Array arguments marked "host or device" may point to either; the library inspects the
 *     pointer.  When any such OUTPUT is in host memory the call blocks until it is filled.
 *     Device outputs are written asynchronously on `stream`.
 *   - The caller owns every buffer it passes; the library owns only what it allocates inside the
 *     context (the loaded samples' sorted copies and cumulative arrays, and the staging and scratch
 *     of the evaluation calls, kept for reuse), and kvdro_destroy() frees that.
 *   - A context belongs to one device and one host thread at a time.
 *   - Ties: the minimum over lam and the argmin over r both take the lowest index.
 */
#ifndef KVDRO_H
#define KVDRO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kvdro_ctx kvdro_ctx;

typedef enum {
    KVDRO_OK = 0,
    KVDRO_EINVAL = -1,   /* bad argument; nothing was launched */
    KVDRO_ENOMEM = -2,   /* a device or pinned-host allocation failed */
    KVDRO_ECUDA = -3,    /* a CUDA call failed (message in kvdro_last_error) */
    KVDRO_ESTATE = -4,   /* call out of order, e.g. eval before samples are loaded */
    KVDRO_ETIMEOUT = -5, /* a kernel gave up a bounded wait and reported it; the outputs are then
                            incomplete (r_idx is -1 where no r was evaluated) */
    KVDRO_ERANGE = -6    /* a page cache kernel met a value in device memory outside its range (a page
                            number, a slot, a length); it left out what the value stood for.  Reported
                            by kvdro_sync */
} kvdro_status;

typedef enum {
    KVDRO_FP32 = 0,      /* FP32 outputs.  When every L_max <= 2^22 they are the KVDRO_EXACT
                            results rounded to FP32 (the exact kernel is also the fastest);
                            otherwise per-term arithmetic in FP32 with sums folded into FP64 */
    KVDRO_FP64 = 1,      /* FP64 outputs.  When every L_max <= 2^22 (and no cost times a class's
                            L_max * N passes 1e300) they are the KVDRO_EXACT results, whose sums
                            carry no rounding; otherwise per-term arithmetic and sums in FP64 */
    KVDRO_EXACT = 2,     /* per term, exact integer arithmetic on exact integer thresholds
                            (|x + 1 - t| summed exactly, four samples at a time); exact integer
                            counts and sums combined once per cell in FP64, so results carry
                            FP64 rounding only.  Needs every L_max <= 2^22. */
    KVDRO_ENVELOPE = 3   /* not per term: each cell's sample sum from the sorted samples'
                            cumulative counts and sums at its exact threshold, O(1) per cell,
                            FP64 outputs with FP64 rounding only */
} kvdro_precision;

/* Create a context on CUDA device `device_ordinal`.  *out receives the handle (NULL on error).
 * Two environment variables, read here, are test hooks and must not be set in production:
 * KVDRO_TEST_FAIL_ALLOC=n makes the context's n-th allocation fail (KVDRO_ENOMEM), and
 * KVDRO_TEST_SKIP_CHUNK=c makes this context's grid kernels leave staged chunk c uncopied with a
 * wait bound of 1 ms, so every bounded wait on it runs out (KVDRO_ETIMEOUT).  The hook travels
 * with this context's launches only; other contexts, on the same device or not, keep the
 * production bound.  kvdro_kv_attend leaves out the c-th copies of each CTA, to the same effect.
 * Bounded waits: a grid kernel gives up waiting for a staged sample chunk only after 2 s of the
 * GPU's global timer AND a minimum number of polls made while it was running, so a CTA that is
 * descheduled (time-slicing, preemption) does not report a timeout on a copy that lands once it
 * resumes. */
int kvdro_create(kvdro_ctx** out, int device_ordinal);

/*
 * Load the per-class empirical samples (the empirical distribution of Sec. 2.4 and the
 * Alg. 1 input) and sort them.  Replaces any previously loaded samples.
 *   K        number of classes, 1 <= K <= 4096.
 *   offsets  host int64[K+1], CSR offsets: offsets[0] = 0, N_k = offsets[k+1] - offsets[k] >= 1,
 *            N_k <= 2^31 - 1.
 *   lengths  host or device int32[offsets[K]], class k's samples at [offsets[k], offsets[k+1]),
 *            each in [0, L_max[k]] (checked on the device; a violation gives KVDRO_EINVAL).
 *   L_max    host int32[K], support upper end L_k, 1 <= L_k <= 2^24.
 *   L_in     host int32[K] input length per class (>= 0, L_in + L_max <= 2^24), or NULL for zeros.
 * Runs the segmented counting sort and the cumulative count arrays on `stream`, then blocks
 * until the range check has been read back.
 */
int kvdro_load_samples(kvdro_ctx* ctx, int32_t K, const int64_t* offsets, const int32_t* lengths,
                       const int32_t* L_max, const int32_t* L_in, void* stream);

/*
 * Lower empirical quantiles of every loaded class: out[k*F + f] = x_(m), the m-th smallest
 * sample of class k, m = max(1, ceil(fractiles[f] * N_k)) computed in FP64.
 *   F          1 <= F <= 65536;  fractiles: host double[F], each in [0, 1].
 *   out        host or device int32[K*F].
 */
int kvdro_quantiles(kvdro_ctx* ctx, int32_t F, const double* fractiles, int32_t* out, void* stream);

/*
 * Evaluate the grid and reduce it.  Element type of S, cost and min_cost is float for
 * KVDRO_FP32 and double for the other modes.
 *   R, r       host int32[R], 1 <= R <= 2^20; every r must satisfy L_in_k <= r <= L_in_k + L_k for
 *              every class (the reservation domain of Sec. 2.2).
 *   NL, lam    host double[NL], finite, >= 0; 1 <= NL <= 256 (128 for KVDRO_FP64).
 *   E, eps     host double[E], finite, >= 0; 1 <= E <= 64.
 *   M, c_p,c_w host double[M] each, finite, >= 0; 1 <= M <= 65536.
 * Outputs (each may be NULL to skip it; host or device).  With M > 1, host S, cost and lam_idx
 * come back in up to 16 blocks of regimes on a stream of the context's own; into page-locked host
 * memory each block's copy overlaps the evaluation of the next (a copy into pageable memory holds
 * the calling thread until it is done, so those blocks alternate with the evaluation instead).
 * The call returns only once every output is filled.
 *   S          [M][K][R][NL]  mean supremum S(eta, lam)
 *   cost       [M][E][K][R]   min over lam of lam*eps + S
 *   lam_idx    int32 [M][E][K][R]  lowest lam index attaining cost
 *   r_idx      int32 [M][E][K]     lowest r index attaining min_r cost
 *   min_cost   [M][E][K]
 *   fhat       double [M][E][K]    #{x <= r* - L_in} / N  (empirical CDF at the chosen r)
 */
int kvdro_eval_grid(kvdro_ctx* ctx, int precision, int32_t R, const int32_t* r, int32_t NL, const double* lam,
                    int32_t E, const double* eps, int32_t M, const double* c_p, const double* c_w, void* S,
                    void* cost, int32_t* lam_idx, int32_t* r_idx, void* min_cost, double* fhat, void* stream);

/*
 * The exact worst-case expected cost, without restricting gamma to a grid: for every regime,
 * radius, class and reservation, min over gamma >= 0 of gamma*eps + S(eta, gamma) (App. A,
 * eq. app_kantorovich; the value of the epigraph LP of eq. app_lp, which equals the worst case
 * over the Wasserstein ball by the strong duality of App. A Step 2).  The objective is convex
 * and piecewise linear in gamma with its minimiser in [0, max(c_p, c_w)]; the library
 * searches on the sign of its right derivative, over the integer thresholds between which it is
 * constant and then over the ordered bit patterns of the nonnegative doubles (down to two adjacent
 * doubles at any scale), with every evaluation O(1) from the sorted samples' cumulative counts and sums, so results carry FP64 rounding only.  The result is
 * never below the empirical cost (1/N) sum_n Q(eta, x_n), computed exactly from integer sums:
 * that bound holds at every gamma (App. A) and is the value itself at eps = 0.
 * Arguments as kvdro_eval_grid; outputs (each may be NULL; host or device):
 *   cost       double [M][E][K][R]   the exact dual value
 *   gamma      double [M][E][K][R]   a minimising gamma
 *   r_idx      int32 [M][E][K]       lowest r index attaining the minimum (among costs equal to
 *                                    2^-32 relative)
 *   min_cost   double [M][E][K];  fhat  double [M][E][K]  as in kvdro_eval_grid
 */
int kvdro_eval_dual(kvdro_ctx* ctx, int32_t R, const int32_t* r, int32_t E, const double* eps, int32_t M,
                    const double* c_p, const double* c_w, double* cost, double* gamma, int32_t* r_idx,
                    double* min_cost, double* fhat, void* stream);

/* Copy the sorted samples (class by class, ascending, int32[offsets[K]]) to `out` (host or device). */
int kvdro_sorted_samples(const kvdro_ctx* ctx, int32_t* out, void* stream);

/*
 * Device time, in milliseconds, of the grid-kernel launches of the last kvdro_eval_grid() or
 * kvdro_eval_dual() call on this context, measured with CUDA events recorded on that call's
 * stream immediately before and after them (the output copies are outside, and so is the argmin
 * finalisation, but for small grids, whose last CTAs do it).  Blocks until the second event has completed.  KVDRO_ESTATE if nothing has been
 * evaluated yet.
 */
int kvdro_last_grid_ms(kvdro_ctx* ctx, float* ms);

/*
 * kvdro_eval_grid_noalloc -- the FP32 grid evaluation (load, sort, grid, argmin) in one call
 * that allocates nothing.  The paper has no counterpart; this entry point exists for callers
 * that cannot allocate device memory at the time they need an answer: a serving engine that
 * has handed all free device memory to its KV-cache block pool at start-up (a new cudaMalloc
 * would fail or evict cache blocks), a process held to a fixed device-memory budget, or a
 * latency-critical loop that must not call cudaMalloc/cudaFree because cudaFree synchronises
 * the whole device.
 *
 * Instead of a context, it works in one static device array of KVDRO_NOALLOC_SCRATCH_BYTES
 * bytes, defined in the library; every GPU that loads the library holds that array until the
 * process exits.  The first call on a device (with that device current) resolves the array's
 * device address, sets kernel attributes and loads every kernel that a call can choose; make that
 * first call while device memory is free for the kernels' code and before any stream capture.
 * Calls share the array: it keeps the last call's contents (the call clears what must start at
 * zero), and calls whose GPU work overlaps in time race on it -- serialise them, e.g. on one
 * stream.  A problem whose scratch would exceed the array (about 12 bytes per sample plus
 * 4 bytes per support point and 8 bytes per (regime, radius, class) row; with more than 128 lam
 * values and every L_max <= 2^22 the limit also counts 12 bytes per (regime, radius, class, r) cell,
 * which the call does not use) is rejected with KVDRO_EINVAL and a
 * message.
 *
 * Arguments are those of kvdro_load_samples and kvdro_eval_grid with precision KVDRO_FP32,
 * on the current device, except that `lengths` and every output must be device memory, there
 * is no S output, and `err` (may be NULL) receives up to err_len bytes of error text.  The
 * call works on `stream` and returns once the outputs are written (it reads the samples' range
 * check and the kernels' status word back), so a grid kernel that gave up a bounded wait is
 * reported here as KVDRO_ETIMEOUT (the outputs are then incomplete).  The test hook
 * KVDRO_TEST_SKIP_CHUNK of kvdro_create is read at every call of this entry point.
 */
#define KVDRO_NOALLOC_SCRATCH_BYTES (32u << 20)
int kvdro_eval_grid_noalloc(int32_t K, const int64_t* offsets, const int32_t* lengths, const int32_t* L_max,
                            const int32_t* L_in, int32_t R, const int32_t* r, int32_t NL, const double* lam,
                            int32_t E, const double* eps, int32_t M, const double* c_p, const double* c_w,
                            float* cost, int32_t* lam_idx, int32_t* r_idx, float* min_cost, double* fhat,
                            void* stream, char* err, int32_t err_len);

/*
 * The page cache -- what a serving engine does with the reservations.  Keys and values live in
 * pages of `page_size` token slots; a request holds a row of page numbers (its block table), as many
 * as its reservation r asks for.  One step of a server is
 *     kvdro_kv_plan     pages for the requests' lengths and reservations, slots for their new tokens
 *     kvdro_kv_append   the new tokens' keys and values into those slots     (once per layer)
 *     kvdro_kv_attend   the new tokens' attention over their requests' pages (once per layer)
 * Where requests share a prefix, kvdro_kv_attend_shared stands in the place of the last; kvdro_kv_read gets keys and values back out of
 * pages.  A cache is of 16 bits (kvdro_kv_open) or of 8 (kvdro_kv_open8); every call takes handles of both.
 * The paper's data plane runs a paged cache of this kind unchanged beneath its decisions (Fig. 1, Sec. 2).
 * All arrays are memory of the context's device (or managed) and every call is asynchronous on `stream` and allocates nothing, so
 * that calls can be captured into a CUDA graph (after one call of the same kind outside a capture,
 * which loads its kernels).  A value in device memory that is out of range is never followed: the kernels leave
 * out what it stands for and the next kvdro_sync() returns KVDRO_ERANGE.
 * Calls on one context may use several streams: kvdro_kv_attend and kvdro_kv_attend_shared order their scratch across
 * them themselves, outside of captures (the launches of captured graphs that share a context must be ordered by
 * the caller); the caller orders everything else (his arrays) as for any kernel.
 */
typedef struct kvdro_kv kvdro_kv;

typedef enum { KVDRO_BF16 = 0, KVDRO_FP16 = 1 } kvdro_kv_dtype;

/*
 * Describe a page cache that the caller owns: k and v hold element (page, slot, head, d) at
 * page * stride[0] + slot * stride[1] + head * stride[2] + d, strides in elements (NULL: [n_pages][page_size]
 * [n_kv_heads][head_dim], contiguous).
 *   dtype       KVDRO_BF16 or KVDRO_FP16;  page_size: 16, 32, 64 or 128;  head_dim: 64 or 128.
 *   n_pages     >= 1, n_pages * page_size < 2^31;  1 <= n_kv_heads <= 1024.
 *   k, v        device memory, 16-byte aligned, strides positive multiples of 8 elements below 2^39.
 * The arrays must outlive the handle; the handle must not be used after kvdro_destroy(ctx), which frees
 * the handles left open.  Allocates scratch of the context's own, at the first call.
 */
int kvdro_kv_open(kvdro_ctx* ctx, kvdro_kv** out, int dtype, int32_t n_pages, int32_t page_size, int32_t n_kv_heads,
                  int32_t head_dim, void* k, const int64_t* k_stride, void* v, const int64_t* v_stride);

/*
 * Describe a page cache of 8 bits.  k and v hold e4m3 codes (one byte per element, strides as in kvdro_kv_open but
 * multiples of 16), k_exp and v_exp a scale byte for every token and key head, at (page * n_kv_heads + head) * page_size + slot:
 * an element stands for its code times 2^(byte - 127).  Bytes are 1 to 254; 0 stands for zeros.
 * kvdro_kv_append quantises as it writes: byte - 127 is the least E >= -126 with max |x_d| <= 448 * 2^E over the head's finite
 * elements, the codes are x_d / 2^E rounded to nearest, ties to even, so that every element is within 2^-4 of itself or 2^(E-10).
 * Non-finite elements become NaN.  With FP16 rows E = 8 stops at 240 * 2^8 = 61440, for 256 * 2^8 is no FP16 number.  BF16 rows have no such
 * stop: an element of 1.9375 * 2^127 or more becomes 2^128, which is an infinity as BF16.
 *   dtype       the type of the rows that calls on the handle take and give (append, read, q, out): KVDRO_BF16 or
 *               KVDRO_FP16.  To a handle of KVDRO_FP16 elements beyond FP16's range (written as BF16) are infinities in kvdro_kv_read and
 *               where many new rows share a key head; attention of few (at most 24) multiplies codes and takes them as they are.
 *   k, v, k_exp, v_exp  device memory, 16-byte aligned.  The rest as in kvdro_kv_open.
 */
int kvdro_kv_open8(kvdro_ctx* ctx, kvdro_kv** out, int dtype, int32_t n_pages, int32_t page_size, int32_t n_kv_heads,
                   int32_t head_dim, void* k, const int64_t* k_stride, uint8_t* k_exp, void* v, const int64_t* v_stride,
                   uint8_t* v_exp);

/* Free the handle (the arrays stay the caller's).  NULL is accepted. */
int kvdro_kv_close(kvdro_kv* kv);

/*
 * Pages for one step.  For request b with cached[b] tokens in the cache, new_len[b] tokens to come in this
 * step, reserve[b] tokens to hold pages for (the reservation r, input included) and held[b] pages at table[b]:
 *   new_len > 0   pages are handed out until ceil(max(cached + new_len, min(reserve, max_pages * page_size)) /
 *                 page_size) are held.  In the order of b, until one does not fit the free pages: that request and every later one
 *                 that needs pages is refused, as is one whose tokens pass max_pages * page_size.  A refused request keeps
 *                 what it holds; its tokens have slot and pos -1 and its kv_len is 0.
 *   new_len = 0   the request waits: it keeps its pages.
 *   new_len < 0   the request is done: its pages go back, to be handed out from the next call on.
 * Free pages are a ring of n_pages page numbers: pool = {head, count}; pages are taken at head and
 * returned behind the last.  Every page number is in the ring or in one request's table.
 *   page_size, n_pages   as in kvdro_kv_open;  1 <= B <= 16384;  max_pages >= 1, max_pages * page_size <= 2^30.
 *   cached, new_len, held  int32[B];  reserve: int32[B] or NULL (no reservations).
 *   table      int32[B][max_pages], updated: entries held[b] <= j < held_out[b] are written.
 *   ring       int32[n_pages], updated: returned pages are written behind the last.  An entry, of a table or of the
 *              ring, that is no page number is a range error each time it is returned or handed out; it stays in the ring, and in
 *              the table of the request that gets it, as -1 (tokens there have slot -1).
 *   pool       int32[2];  pool_out: int32[2];  held_out: int32[B] (held and pool are not changed: the same
 *              call again gives the same results).
 *   q_off      int32[B+1]  prefix sums of max(new_len, 0): request b's tokens are q_off[b] .. q_off[b+1]-1.
 *   kv_len     int32[B]    cached + new_len, the tokens that kvdro_kv_attend sees; 0 if refused or done.
 *   slot, pos  int32[T] (pos may be NULL; T >= 0)  page * page_size + offset, and the position in the request, of every
 *              new token; -1 behind the last token.  More new tokens than T is a range error (the rest is left out).
 * No array that is written (kv_len over cached, say) may overlap another of the call: KVDRO_EINVAL.
 */
int kvdro_kv_plan(kvdro_ctx* ctx, int32_t page_size, int32_t n_pages, int32_t B, int32_t max_pages, int32_t T,
                  const int32_t* cached, const int32_t* new_len, const int32_t* reserve, const int32_t* held,
                  int32_t* table, int32_t* ring, const int32_t* pool, int32_t* held_out, int32_t* pool_out,
                  int32_t* q_off, int32_t* kv_len, int32_t* slot, int32_t* pos, void* stream);

/*
 * Write T tokens' keys and values into their slots: cache[slot[t]] = k[t], v[t] for every head; a
 * token whose slot is -1 is skipped.  Slots must differ from one another.
 *   k, v       element (t, head, d) at t * stride[0] + head * stride[1] + d, strides in elements (NULL: contiguous
 *              [T][n_kv_heads][head_dim]), of the cache's dtype; 16-byte aligned, strides multiples of 8.
 *   slot       int32[T], T >= 0.
 */
int kvdro_kv_append(kvdro_kv* kv, int32_t T, const void* k, const int64_t* k_stride, const void* v,
                    const int64_t* v_stride, const int32_t* slot, void* stream);

/*
 * Read keys and values back out of pages: those of the last n = q_off[b+1] - q_off[b] tokens of request b's kv_len[b], so that with
 * the arrays of a step it gives what kvdro_kv_append wrote in it, and with n = kv_len[b] whole requests.
 *   q_off, kv_len, table, B, T, max_pages   as in kvdro_kv_attend.
 *   k, v       results, element (t, head, d) at t * stride[0] + head * stride[1] + d (NULL: contiguous [T][n_kv_heads]
 *              [head_dim]), of the handle's dtype, rounded to it once (8 bits); 16-byte aligned, strides multiples of 8.  Tokens of no
 *              request, in front of position 0 and on pages that are none get zeros.
 */
int kvdro_kv_read(kvdro_kv* kv, int32_t B, int32_t T, const int32_t* q_off, const int32_t* kv_len, const int32_t* table,
                  int32_t max_pages, void* k, const int64_t* k_stride, void* v, const int64_t* v_stride, void* stream);

/*
 * Attention of the new tokens over their requests' cached ones, their own included (append first).  Token i
 * of request b's n = q_off[b+1] - q_off[b] stands at position p = kv_len[b] - n + i; its query head h reads key/value
 * head h / (n_heads / n_kv_heads):
 *     out = sum_j softmax_j(s_j) v_j,   s_j = f(scale q . k_j),   f(x) = x, or softcap tanh(x / softcap)
 * over the positions j < kv_len[b] with j <= p (causal) and j > p - window (window > 0).  A token that sees
 * no position gets out = 0 and lse = -infinity.  What is stored at unseen positions does not
 * matter, NaN included, nor do the table's entries of pages that no token of the request sees (behind a window, say).
 * Products are of the cache's dtype with FP32 sums (scores below 2^120: a query's largest element times a key's times the scale); the softmax is
 * FP32, its weights are rounded to the cache's dtype for the product with v.  That product's sums are FP32 of weights of up to 2^8 and divided at
 * the end, so that values above 2^120 / (positions seen) may pass FP32 in them.
 * Over 8 bits few tokens (up to 24 rows that share a key head) are multiplied as FP16: codes as they are, BF16 queries off by 2^-25 of their row's
 * largest element at most, and weights times a power of two, w_j 2^(E_j), of which what is below 2^-32 of a row's largest is lost.  Their sums are no
 * larger than the values.
 *   B          requests, 1 <= B <= 16384;  T: tokens, T >= 0; tokens beyond T are left out, and T tokens of out and lse
 *              are written (zeros and -infinity for tokens of no request).
 *   n_heads    a multiple of n_kv_heads, at most 4096; T * n_heads <= 2^30.
 *   max_q      the most new tokens of one request, as far as the caller knows, 0 if unknown.  It chooses among
 *              kernels; the results are right whatever it says.
 *   q, out     element (t, h, d) at t * stride[0] + h * stride[1] + d (NULL: contiguous [T][n_heads][head_dim]), of the
 *              cache's dtype; 16-byte aligned, strides multiples of 8.
 *   q_off      int32[B+1], ascending from 0;  kv_len: int32[B];  table: int32[B][max_pages], max_pages * page_size <= 2^30.
 *   scale      finite;  causal: 0 or 1;  window >= 0 (0: none; needs causal);  softcap 0 (none) or in
 *              [2^-20, 1000]; capped scores are off by up to 2^-20 softcap, also where they are small.
 *   lse        float [T][n_heads], log sum_j exp(s_j); may be NULL.
 */
int kvdro_kv_attend(kvdro_kv* kv, int32_t B, int32_t T, int32_t n_heads, int32_t max_q, const void* q,
                    const int64_t* q_stride, const int32_t* q_off, const int32_t* kv_len, const int32_t* table,
                    int32_t max_pages, double scale, int causal, int32_t window, double softcap, void* out,
                    const int64_t* out_stride, float* lse, void* stream);

/*
 * Attention of requests that share prefixes: requests share_off[g] .. share_off[g+1] - 1 stand behind the same prefix_len[g]
 * tokens, which live once in the pages prefix_table[g]; kv_len and table are about a request's own tokens alone (as kvdro_kv_plan gives
 * them).  A token sees what kvdro_kv_attend lets it see of its own tokens, and the whole prefix: the softmax runs over both.
 * A prefix is read once for all of its requests' tokens, whose rows it makes one long request of; where few requests stand behind short ones
 * (prefix_pages says how long they may be) each reads its own, which is faster.  Tokens of requests with
 * kv_len 0 get out = 0 and lse = -infinity, prefix or not.  There is no sliding window.
 *   G            prefixes, 1 <= G <= B;  share_off: int32[G+1], ascending within [0, B]: requests in front of the first and
 *                behind the last have no prefix.
 *   prefix_len   int32[G], 0: none;  prefix_table: int32[G][prefix_pages], prefix_pages * page_size <= 2^30.
 *   work         device memory of the bytes that kvdro_kv_shared_bytes gives for these sizes, 16-byte aligned: scratch of this call until
 *                its work is done on the device, to be used by any other call after it.
 * The other arguments are those of kvdro_kv_attend, max_q the most new tokens of one request.
 */
int kvdro_kv_attend_shared(kvdro_kv* kv, int32_t B, int32_t T, int32_t n_heads, int32_t max_q, const void* q,
                           const int64_t* q_stride, const int32_t* q_off, const int32_t* kv_len, const int32_t* table,
                           int32_t max_pages, int32_t G, const int32_t* share_off, const int32_t* prefix_len,
                           const int32_t* prefix_table, int32_t prefix_pages, double scale, int causal, double softcap, void* out,
                           const int64_t* out_stride, float* lse, void* work, size_t work_bytes, void* stream);

/* Bytes of `work` for T tokens.  KVDRO_EINVAL outside the limits of kvdro_kv_attend. */
int kvdro_kv_shared_bytes(int32_t T, int32_t n_heads, int32_t head_dim, size_t* bytes);

/* Wait for the context's device work -- the streams of its last call outside the page cache and of its last page cache
 * call, and its last kvdro_kv_attend or kvdro_kv_attend_shared -- and report any asynchronous CUDA error, kernel timeout or value out
 * of range.  (Earlier page cache calls on yet other streams: what their kernels found is reported once they are
 * done.) */
int kvdro_sync(kvdro_ctx* ctx);

/* Text of the last error on this context ("" if none).  Valid until the next call on ctx. */
const char* kvdro_last_error(const kvdro_ctx* ctx);

/* Free the context and everything it owns.  NULL is accepted. */
int kvdro_destroy(kvdro_ctx* ctx);

#ifdef __cplusplus
}
#endif

#endif /* KVDRO_H */
