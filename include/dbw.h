/*
 * dbw.h -- C ABI of the Dynamic Backup Workers (DBW) hot path on one MI355X.
 *
 * The library simulates a synchronous parameter server (PS) with n logical
 * workers on one GPU (Xu, Neglia, Sebastianelli, "Dynamic Backup Workers for
 * Parallel Machine Learning", Sect. 2 and Sect. 3):
 *   - every worker computes a minibatch gradient at the same w_t (Eq. gradient);
 *   - the PS averages only the k_t fastest gradients (Eq. grad_bw) and updates
 *     w (Eq. update);
 *   - DBW picks k_t = n - b_t from end-of-iteration gradient statistics
 *     (Eqs. sumvariancekt, normsquarekt, estimateL and their D-window means,
 *     Eq. gain) and from an estimate of the order-statistic arrival times
 *     (Eq. quadratic_opt), maximising gain per unit of time (Eqs. greedy,
 *     greedy2).
 *
 * Conventions for every entry point:
 *   - Pointers named as DEVICE are device memory owned by the caller; they are
 *     read or written asynchronously on the context's HIP stream and must stay
 *     valid until the stream has passed the call.  HOST pointers are read or
 *     written before the call returns.
 *   - Arrays are dense and row-major; float is IEEE fp32, double fp64.
 *   - Model parameters w have P = dbw_param_count(cfg) floats:
 *       softmax regression: W [d][C] (no bias), P = d*C;
 *       MLP d-H-C with ReLU: [W1 (d x H) | b1 (H) | W2 (H x C) | b2 (C)];
 *       CNN: [W1 (800 x H) | b1 (H) | W2 (H x C) | b2 (C) | Wc1 (20 x 1 x 5 x 5) |
 *       bc1 (20) | Wc2 (50 x 20 x 5 x 5) | bc2 (50)], P = 800 H + H + H C + C + 25570.
 *     Gradients use the same layout.
 *   - Every call returns a dbw_status; nothing throws across the ABI.  Argument
 *     errors are detected on the host before any work is queued (DBW_EINVAL,
 *     DBW_ERANGE).  Errors only the kernels can see (a minibatch row index
 *     outside the dataset, k larger than the number of workers that ever
 *     arrive) raise a device error flag that dbw_sync() reports.  HIP failures
 *     return DBW_EHIP.  dbw_last_error() gives a text for the last failure.
 *   - A context is not thread-safe; distinct contexts are independent.
 */
#ifndef DBW_H
#define DBW_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DBW_OK = 0,
  DBW_EINVAL = -1,      /* bad argument: NULL pointer, shape, config        */
  DBW_ERANGE = -2,      /* k outside [1, n] or beyond the workers that arrive,
                           row index outside the dataset                     */
  DBW_EHIP = -3,        /* a HIP runtime call failed                         */
  DBW_ESTATE = -4,      /* call does not fit the context's state             */
  DBW_EUNSUPPORTED = -5 /* shape the kernels do not handle                   */
} dbw_status;

/* DBW_CNN: the MNIST network shape of Sect. 4 (two 5 x 5 convolutions and
 * two fully connected layers) on 28 x 28 single-channel images (d = 784):
 * conv 1 -> 20 channels, 2 x 2 max pooling, ReLU, conv 20 -> 50, 2 x 2 max
 * pooling, ReLU, the 800 features (channel, row, column), FC 800 -> H with
 * ReLU, FC H -> C.  Convolutions are valid, stride 1; a pooling window passes
 * (and back-propagates to) its first largest entry in row-major order. */
typedef enum { DBW_SOFTMAX = 0, DBW_MLP = 1, DBW_CNN = 2 } dbw_model;

/* Virtual clock of the simulated cluster (Sect. 2, the synchronisation
 * variants; Sect. 3.2).  FRESH: every worker starts each iteration at its
 * beginning, so a worker's arrival offset is its round-trip time and all n
 * arrivals are samples.  PSW (Push & Wait): the PS pushes w_{t+1} once it
 * holds k_t gradients of w_t; a worker still computing a gradient of an older
 * vector finishes it, then takes the most recent vector; with s_t the start
 * of iteration t and b_i the time worker i becomes free, worker i computes
 * w_t iff b_i <= s_t or b_i < s_{t+1}, its offset is
 * max(s_t, b_i) - s_t + tau_i, and a worker still busy at s_{t+1} skips w_t
 * (no sample: the estimate's data are censored).  PSI (Push & Interrupt):
 * the PS pushes w_{t+1} once it holds k_t gradients of w_t and every worker
 * drops the gradient it is computing to start on w_{t+1}; offsets are the
 * round-trip times as under FRESH, but only the first k_t arrivals in
 * (offset, worker index) order complete, so only they are samples. */
typedef enum { DBW_CLOCK_FRESH = 0, DBW_CLOCK_PSW = 1, DBW_CLOCK_PSI = 2 } dbw_clock;

/* How k_t is chosen (Sect. 3.3; the settings compared in Sect. 4).
 * DBW: Eqs. gain, greedy, greedy2.  STATIC: k_t = k_static at every
 * iteration (a fixed number of backup workers); the objective is still
 * computed as under DBW.  BLIND (B-DBW): the gain G_k is replaced by k and
 * the rest of the rule is unchanged (k_t = n before the first smoothness
 * estimate, the largest k among equal objectives, the loss guard). */
typedef enum { DBW_POLICY_DBW = 0, DBW_POLICY_STATIC = 1, DBW_POLICY_BLIND = 2 } dbw_policy;

/* Time estimate T_hat_k (Sect. 3.2).  ISOTONIC: from the solution of Eq.
 * quadratic_opt (see dbw_time_estimate).  NAIVE: the empirical mean of the
 * samples of cell (k,k), the first approach the section sets aside; NaN (k
 * not eligible) while that cell holds no sample. */
typedef enum { DBW_ESTIMATOR_ISOTONIC = 0, DBW_ESTIMATOR_NAIVE = 1 } dbw_estimator;

/* Rows of the worker-gradient buffer that dbw_step writes (the PS only uses
 * the k_t fastest gradients, Eq. grad_bw).  ALL: every worker's row (the
 * aggregation then reads the selected ones back).  SELECTED: only the
 * selected workers' rows; NONE: no row is asked for.  With SELECTED or NONE,
 * wherever the softmax gradients take the single pass (see dbw_grads_route)
 * with several row slabs a worker, one kernel sums the selected workers' slab
 * partials and aggregates them directly, so the unselected rows are never
 * formed and no row is read back; g_t, the updated w, the losses, k and the
 * mask are bitwise those of ALL, the statistics equal up to the order of their
 * fp64 and fp32 partial sums.  Where the gradients come from per-worker GEMM
 * tiles and P > 131072 (softmax under SELECTED or NONE, the MLP and the CNN
 * under SELECTED), the choice and the selection run before the gradient
 * kernels, which compute every worker's gradient but store only the selected
 * rows; k, the mask, g_t, w, the losses and the statistics are bitwise those
 * of ALL.  With smaller P every row is formed before the choice: softmax of up
 * to 16 classes under SELECTED keeps them in a second buffer of n*P floats,
 * from which the selected rows are copied; elsewhere G itself holds them, also
 * under NONE.  Rows not written hold unspecified values after dbw_step.
 * dbw_worker_grads always writes every row. */
typedef enum { DBW_G_ROWS_ALL = 0, DBW_G_ROWS_SELECTED = 1, DBW_G_ROWS_NONE = 2 } dbw_g_rows;

#define DBW_MAX_N 1024 /* logical workers per context                       */
#define DBW_MAX_D 64   /* length of the estimator averaging window D          */

/* Problem description.  n workers, minibatch B per worker, d input features,
 * C classes, H hidden units (MLP only), learning rate eta (constant for all
 * k), window D of the estimator averages, loss guard factor beta >= 1
 * (Eq. greedy2), virtual clock (dbw_clock; 0 = fresh start), rule of the
 * choice of k (dbw_policy; 0 = DBW) and time estimate (dbw_estimator; 0 =
 * isotonic), rows of G that dbw_step writes (dbw_g_rows; 0 = all).
 * Zero-initialised fields give the method as defined.  S > 0 declares
 * a resident dataset of S rows that minibatches may index (see
 * dbw_worker_grads); S = 0 means minibatches are passed materialised. */
typedef struct {
  int32_t model; /* dbw_model */
  int32_t n, B, d, C, H;
  int32_t D;
  int32_t clock;     /* dbw_clock */
  int32_t policy;    /* dbw_policy */
  int32_t k_static;  /* k of DBW_POLICY_STATIC, in [1, n]; ignored otherwise */
  int32_t estimator; /* dbw_estimator */
  int32_t g_rows;    /* dbw_g_rows */
  double eta, beta;
  int64_t S;
} dbw_config;

/* End-of-iteration statistics over the k received gradients (Sect. 3.1):
 * gnorm2 = ||g_t||^2; V_plus = Eq. sumvariancekt (for k = 1 the current
 * D-window mean of past V_plus, 0 without history); N_plus = Eq.
 * normsquarekt; F_hat = mean minibatch loss of the received workers. */
typedef struct {
  double gnorm2, V_plus, N_plus, F_hat;
} dbw_iter_stats;

/* DBW estimator state carried between iterations (Sect. 3.1, 3.3).  Histories
 * are oldest first; only the last D entries are kept.  hL holds the
 * smoothness estimates L_plus (Eq. estimateL), pushed from the second
 * iteration on when their denominator is positive.  F_prev, F_prev2 are
 * F_hat of the two previous iterations (nF of them valid). */
typedef struct {
  int64_t t;      /* iterations completed                                   */
  int32_t k_prev; /* k_{t-1}; n before the first iteration                  */
  int32_t nV;     /* valid entries of hV and hN                              */
  int32_t nL;     /* valid entries of hL                                     */
  int32_t nF;     /* valid entries among F_prev, F_prev2 (0..2)              */
  double F_prev, F_prev2;
  double hV[DBW_MAX_D], hN[DBW_MAX_D], hL[DBW_MAX_D];
} dbw_estimator_state;

typedef struct dbw_ctx dbw_ctx;

/* P for a configuration; -1 if the configuration is invalid. */
int64_t dbw_param_count(const dbw_config* cfg);

/* The kernels that dbw_worker_grads and dbw_step run for the softmax gradients
 * of cfg (diagnostics; HOST only, needs no device).  single_pass: 1 if one
 * kernel reads X once (up to 16 classes), 0 if logits and gradient are two
 * products; slabs: row slabs of a worker whose partial gradients are summed
 * (single pass; else 1); per_row: 1 if minibatches given by `rows` share the
 * logits of the dataset's rows.  (0, 1, 0) for the MLP and the CNN.
 * DBW_EINVAL for an invalid cfg or a NULL pointer. */
dbw_status dbw_grads_route(const dbw_config* cfg, int32_t* single_pass, int32_t* slabs, int32_t* per_row);

/* Create a context bound to HIP stream `stream` (a hipStream_t, NULL for the
 * default stream) on the current device.  Validates cfg (n in [1, DBW_MAX_N],
 * B, d, C >= 1, C <= 4096, H >= 1 for the MLP and the CNN, d = 784 for the
 * CNN, D in [1, DBW_MAX_D], eta > 0,
 * beta >= 1, S >= 0), allocates all device workspace (no allocation happens in
 * later calls) and sets the estimator state to its initial value.  Returns
 * DBW_EUNSUPPORTED when one array the kernels address (P floats, the n*B*d
 * minibatch floats, the S*d dataset floats, n*B*C or n*B*H activations)
 * would reach 2 GiB.  Beside G, the workspace of the softmax's two products
 * holds the residuals as matrix-core fragments, 6 bytes a value with every
 * worker's rows padded to 32 and the classes to 16 (n = 1024, B = 1, C = 4096:
 * 805 MB), W likewise, and S*C floats where the dataset's rows share their
 * logits; the MLP's and the CNN's hidden gradients are held the same way. */
dbw_status dbw_create(const dbw_config* cfg, void* stream, dbw_ctx** out);
void dbw_destroy(dbw_ctx* ctx);
/* Text of the last failure on ctx; with ctx NULL, of the last failed
 * context-free call (dbw_grad_stats_static) on the calling thread. */
const char* dbw_last_error(const dbw_ctx* ctx);

/* Waits for the context's stream and reports device-side errors raised since
 * the last dbw_sync (then clears them): DBW_ERANGE for a row index outside
 * [0, S) or k beyond the number of workers whose tick is below INT64_MAX. */
dbw_status dbw_sync(dbw_ctx* ctx);

/* Worker gradients (Sect. 2, Eq. gradient).  For each worker i, at the common
 * parameters w (DEVICE float [P]):
 *   G[i] = (1/B) sum_b grad f(x_{i,b}, w)   (DEVICE float [n][P], out)
 *   loss[i] = (1/B) sum_b f(x_{i,b}, w)      (DEVICE float [n], out)
 * with f the natural-log cross-entropy of the softmax of the model output.
 * Minibatches: if rows == NULL, X is DEVICE float [n][B][d] and y DEVICE int32
 * [n][B]; else X is the resident dataset DEVICE float [S][d], y its labels
 * DEVICE int32 [S], and rows DEVICE int32 [n][B] lists each worker's row
 * indices into it.  Labels must lie in [0, C).  w, X and G must be 16-byte
 * aligned (DBW_EINVAL otherwise).  With rows, all S rows of X and y may be
 * read, also those in no minibatch (their values do not matter and their
 * labels are not checked): none may be written meanwhile.  Where the
 * dataset's rows share their logits (dbw_grads_route), the same minibatches
 * passed materialised give results that agree to fp32 rounding; elsewhere they
 * give the same bits. */
dbw_status dbw_worker_grads(dbw_ctx* ctx, const float* w, const float* X, const int32_t* y,
                            const int32_t* rows, float* G, float* loss);

/* Fastest-k aggregation (Sect. 2, Eq. grad_bw).  ticks (DEVICE int64 [n]) are
 * the round-trip times of the n workers in integer ticks; arrival order is the
 * order of (tick, worker index).  Writes mask (DEVICE uint8 [n]): 1 for the k
 * first arrivals, else 0; and g (DEVICE float [P]) = (1/k) sum of their rows
 * of G (DEVICE float [n][P]).  k (host) must lie in [1, n]. */
dbw_status dbw_aggregate_fastest(dbw_ctx* ctx, const float* G, const int64_t* ticks, int32_t k,
                                 float* g, uint8_t* mask);

/* Gradient statistics over the workers with mask[j] = 1 (Sect. 3.1,
 * Eqs. sumvariancekt, normsquarekt, loss estimate).  G DEVICE float [n][P],
 * mask DEVICE uint8 [n] with exactly k ones, g DEVICE float [P] their mean,
 * loss DEVICE float [n].  Writes sqnorm (DEVICE float [n]) = ||G[j]||^2 for
 * selected j, 0 otherwise, and *stats (DEVICE dbw_iter_stats).  For k = 1
 * V_plus is the context's current D-window mean of V_plus. */
dbw_status dbw_grad_stats(dbw_ctx* ctx, const float* G, const uint8_t* mask, int32_t k,
                          const float* g, const float* loss, float* sqnorm,
                          dbw_iter_stats* stats);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the
 * statistics of dbw_grad_stats with no context, computed by the same kernels
 * on the stream `stream` (a hipStream_t, NULL for the default stream) of the
 * current device.  The call allocates nothing: its scratch (n*ceil(P/256)
 * per-row float and 2*ceil(P/256) per-tile double partial sums, each part
 * rounded up to 256 bytes) lives in one file-scope device array of
 * DBW_STATIC_SCRATCH_BYTES per GPU, held until the process ends.  G DEVICE
 * float [n][P], mask DEVICE uint8 [n], g DEVICE float [P], loss DEVICE float
 * [n]; writes sqnorm (DEVICE float [n]) and *stats (DEVICE dbw_iter_stats) as
 * dbw_grad_stats does, except that for k = 1 V_plus is V_window (HOST, the
 * caller's D-window mean of past V_plus).  A mask that does not hold exactly
 * k ones yields NaN statistics.  Errors: DBW_EINVAL (n outside [1,
 * DBW_MAX_N], P < 1, a NULL pointer, V_window not finite), DBW_ERANGE (k
 * outside [1, n]), DBW_EUNSUPPORTED (P above 2^29, or a scratch need above
 * DBW_STATIC_SCRATCH_BYTES), DBW_EHIP; dbw_last_error(NULL) then gives the
 * text, per calling thread.  Every call on one GPU uses the same array: calls
 * that overlap on one GPU (other streams, other threads) race and must be
 * ordered by the caller.  No part of the array needs clearing between calls
 * (each value a call reads was written earlier in that call). */
#define DBW_STATIC_SCRATCH_BYTES (8u * 1024u * 1024u)
dbw_status dbw_grad_stats_static(int32_t n, int64_t P, const float* G, const uint8_t* mask, int32_t k,
                                 const float* g, const float* loss, double V_window, float* sqnorm,
                                 dbw_iter_stats* stats, void* stream);

/* Choice of k_t = n - b_t from the context's estimator state (Sect. 3.3,
 * Eqs. gain, greedy, greedy2).  T_hat (DEVICE double [n]) holds the time
 * estimates T_hat_k for k = 1..n; an entry that is not finite and positive
 * makes that k ineligible.  Writes k_out, b_out (DEVICE int32) and, if not
 * NULL, objective (DEVICE double [n]) = G_hat_k / T_hat_k (NaN before the
 * first smoothness estimate exists, and for ineligible k).  The state is not
 * modified. */
dbw_status dbw_choose_b(dbw_ctx* ctx, const double* T_hat, int32_t* k_out, int32_t* b_out,
                        double* objective);

/* One full DBW iteration t: estimate T_hat from the arrival times recorded so
 * far (host, Eq. quadratic_opt), choose k_t, compute all n worker gradients,
 * aggregate the k_t first arrivals, compute the statistics, update
 * w <- w - eta g_t (w DEVICE float [P], 16-byte aligned, in place), and push the estimator
 * state.  X, y, rows as in dbw_worker_grads.  ticks_host (HOST int64 [n],
 * >= 0) are the round-trip ticks tau_i of the gradient each worker computes
 * next; the context's clock turns them into arrival offsets (equal to them
 * under DBW_CLOCK_FRESH; under DBW_CLOCK_PSW the call first waits for k_{t-1}
 * and the offsets must stay below 2^48).  The k_t smallest offsets (ties to
 * the lower worker index) are aggregated; once k_t is known the offsets of
 * the workers that compute w_t are recorded, in arrival order, as samples of
 * row h = k_{t-1}, and the virtual clock advances by the k_t-th smallest
 * offset.  If k_host is not NULL the call waits for the iteration's choice and
 * stores k_t there; otherwise it returns as soon as the work is queued. */
dbw_status dbw_step(dbw_ctx* ctx, float* w, const float* X, const int32_t* y,
                    const int32_t* rows, const int64_t* ticks_host, int32_t* k_host);

/* Device views of the buffers the last dbw_step wrote (valid until the next
 * dbw_step on this context): G [n][P], loss [n], g [P], mask [n], sqnorm [n],
 * stats, T_hat [n], objective [n], k, b. */
typedef struct {
  const float* G;
  const float* loss;
  const float* g;
  const uint8_t* mask;
  const float* sqnorm;
  const dbw_iter_stats* stats;
  const double* T_hat;
  const double* objective;
  const int32_t* k;
  const int32_t* b;
} dbw_step_buffers;
dbw_status dbw_step_outputs(dbw_ctx* ctx, dbw_step_buffers* out);

/* Estimate of E[T_{k,k}] for k = 1..n (Sect. 3.2, Eq. quadratic_opt); pure
 * host computation.  cnt and tsum (HOST int64 [n][n], index [h-1][k-1]) are
 * the number and sum (in ticks) of arrival-time samples of the k-th arrival
 * when the previous iteration waited for h gradients.  The estimates solve the
 * constrained least-squares problem exactly; since unsampled cells leave the
 * solution non-unique, T_hat_k (HOST double [n], out) is the smallest value
 * x_{k,k} takes in a feasible completion of the optimum (equal to x*_{k,k}
 * when cell (k,k) was sampled), and NaN when no sampled cell lies below
 * (k,k).  Returns DBW_EINVAL for n outside [1, DBW_MAX_N], negative counts or
 * sums, or a sum on a cell with zero count. */
dbw_status dbw_time_estimate(int32_t n, const int64_t* cnt, const int64_t* tsum, double* T_hat);

/* The same estimate kept across calls (pure host computation).  A caller that
 * re-estimates after adding a few samples per call (one iteration's arrivals)
 * gets the exact result of dbw_time_estimate at a fraction of the cost: the
 * previous solution is re-certified against the new samples and only the
 * parts that stop being optimal are re-solved.  dbw_step uses one of these
 * inside every context.  Same arguments and errors as dbw_time_estimate. */
typedef struct dbw_time_estimator dbw_time_estimator;
dbw_status dbw_time_estimator_create(dbw_time_estimator** out);
void dbw_time_estimator_destroy(dbw_time_estimator* est);
dbw_status dbw_time_estimator_solve(dbw_time_estimator* est, int32_t n, const int64_t* cnt,
                                    const int64_t* tsum, double* T_hat);
/* How the estimator's solves so far were obtained (diagnostics; HOST int64
 * outs, each may be NULL): fast = exact per-column fits that satisfied every
 * other relation of Eq. quadratic_opt, warm = re-certified and repaired
 * previous solutions, full = solves from scratch.  A solve with no sampled
 * cell counts in none of them.  DBW_EINVAL for a NULL estimator. */
dbw_status dbw_time_estimator_stats(const dbw_time_estimator* est, int64_t* fast, int64_t* warm, int64_t* full);

/* Estimator state transfer (resume, lockstep testing).  HOST structs; both
 * calls synchronise the context's stream. */
dbw_status dbw_state_export(dbw_ctx* ctx, dbw_estimator_state* out);
dbw_status dbw_state_import(dbw_ctx* ctx, const dbw_estimator_state* in);

/* Arrival-time samples (HOST int64 [n][n] each, as in dbw_time_estimate) and
 * the virtual clock (HOST int64, ticks).  Export first folds in every
 * iteration whose row is known (it synchronises the stream).  Import also
 * marks every worker idle at the imported clock (DBW_CLOCK_PSW). */
dbw_status dbw_samples_export(dbw_ctx* ctx, int64_t* cnt, int64_t* tsum, int64_t* clock);
dbw_status dbw_samples_import(dbw_ctx* ctx, const int64_t* cnt, const int64_t* tsum,
                              int64_t clock);

/* Push & Wait clock: the time each worker becomes free (HOST int64 [n],
 * ticks on the virtual clock).  Export folds like dbw_samples_export; import
 * replaces the times (each >= 0; DBW_EINVAL otherwise).  Resume and lockstep
 * testing. */
dbw_status dbw_busy_export(dbw_ctx* ctx, int64_t* busy);
dbw_status dbw_busy_import(dbw_ctx* ctx, const int64_t* busy);

/* Kernel timing with HIP events on the streams the kernels run on.  With
 * dbw_profile_enable(ctx, 1) every launch of the device groups is bracketed
 * by events and the host groups accumulate wall-clock host time (steady
 * clock); with 2 only the host groups are kept (no events are recorded, so
 * the host timings are not inflated by them); 0 turns both off.
 * dbw_kernel_time synchronises and returns the summed milliseconds and the
 * count since the last reset.  Host groups: the time-estimate solve, the
 * whole dbw_step call, the part of it spent waiting for the estimate worker,
 * and the part spent queueing GPU work. */
typedef enum {
  DBW_KT_GRADS = 0,
  DBW_KT_AGGREGATE = 1,
  DBW_KT_CHOOSE = 2,
  DBW_KT_HOST_ESTIMATE = 3,
  DBW_KT_HOST_STEP = 4,
  DBW_KT_HOST_WAIT = 5,
  DBW_KT_HOST_QUEUE = 6,
  DBW_KT_COUNT = 7
} dbw_kernel_group;
dbw_status dbw_profile_enable(dbw_ctx* ctx, int32_t mode);
dbw_status dbw_kernel_time(dbw_ctx* ctx, int32_t group, double* total_ms, int64_t* launches);
dbw_status dbw_profile_reset(dbw_ctx* ctx);

/* ---------------------------------------------------------------------------
 * Operators for language models: what a simulation whose workers hold ragged
 * minibatches of tokens, and whose parameters are a language model's, needs
 * beside the calls above.  A layer with weights W_i [d][C] maps T token rows,
 * sorted by group, to T rows of C values; a group is a worker with its own
 * minibatch, or an expert.  The worker gradients G [n][d][C] of these calls
 * are what dbw_aggregate_fastest and dbw_grad_stats_static take.
 *
 * The calls need no context.  They run on `stream` (a hipStream_t, NULL for
 * the default stream) of the current device, allocate nothing, and can be
 * captured into a HIP graph.  offsets (DEVICE int32 [n+1], non-decreasing, in
 * [0, T]) give the rows offsets[i] .. offsets[i+1]-1 of group i; a group may
 * be empty.  Rows before offsets[0] and from offsets[n] on belong to no group:
 * they are not read, and rows of an output there are left as they were.
 * (Offsets that break these rules never lead outside the arrays: each is
 * taken as the nearest allowed value; the results are then unspecified.)
 * Errors: DBW_EINVAL, DBW_EUNSUPPORTED, DBW_EHIP; dbw_last_error(NULL) then
 * gives the text, per calling thread. */
typedef enum { DBW_F32 = 0, DBW_BF16 = 1, DBW_F16 = 2 } dbw_dtype;

/* Products of ragged groups:
 *   FORWARD      Y[t]  = X[t] W_i         (a = X, b = W, out = Y  [T][C])
 *   INPUT_GRAD   dX[t] = dY[t] W_i^T      (a = dY, b = W, out = dX [T][d])
 *   WEIGHT_GRAD  G_i = sum_t X[t]^T dY[t] (a = X, b = dY, out = G [n][d][C];
 *                zero for an empty group)
 * for the rows t of group i.  Inputs are bf16 or fp16 (dtype), the output is
 * of their type or fp32 (out_dtype); sums are held in fp32 and rounded once.
 * ld_d and ld_C are the row strides, in elements, of the arrays [T][d] (X or
 * dX) and [T][C] (Y or dY), ld_W that of every W_i or G_i (>= C), and st_W the
 * distance of W_{i+1} from W_i.  st_W = 0, for FORWARD and INPUT_GRAD only,
 * gives all groups the same W.  Every stride and pointer that is a multiple
 * of 16 bytes, with d and C multiples of 8, makes the loads wide; others are
 * slower.  NaN and infinities of one group's rows never reach another's. */
typedef enum { DBW_GROUP_FORWARD = 0, DBW_GROUP_INPUT_GRAD = 1, DBW_GROUP_WEIGHT_GRAD = 2 } dbw_group_form;
typedef struct {
  int32_t form;      /* dbw_group_form                                       */
  int32_t dtype;     /* DBW_BF16 or DBW_F16                                  */
  int32_t out_dtype; /* dtype or DBW_F32                                     */
  int32_t n;         /* groups, in [1, DBW_MAX_N]                            */
  int32_t d, C;      /* in [1, 2^20]                                         */
  int64_t T;         /* rows, in [0, 2^31)                                   */
  int64_t ld_d, ld_C, ld_W; /* row strides, below 2^21                       */
  int64_t st_W;
} dbw_group_shape;

/* Bytes of workspace that dbw_group_product needs for a shape (HOST out; 0
 * where the work is not split over a long sum).  Needs no device. */
dbw_status dbw_group_workspace(const dbw_group_shape* shape, int64_t* bytes);

/* One product.  offsets, a, b, out and workspace are DEVICE; out must not
 * overlap the inputs (DBW_EINVAL where it is one of them), and rows (or G_i) of
 * out must not overlap each other.  workspace holds at least
 * dbw_group_workspace bytes, 16-byte aligned (NULL where that is 0); its
 * contents need no clearing and are used up when the call is done: calls that
 * may run at the same time need their own. */
dbw_status dbw_group_product(const dbw_group_shape* shape, const int32_t* offsets, const void* a, const void* b,
                             void* out, void* workspace, int64_t workspace_bytes, void* stream);

/* Mean cross entropy of each worker's tokens, and its gradient.  Z (DEVICE
 * [T][C] of dtype, row stride ld_Z elements) are logits, y (DEVICE int32 [T])
 * labels; a negative label masks its row (padding, prompt tokens): its logits
 * are not read, it adds nothing and its gradient is zero.  With count_i the
 * rows of worker i that are not masked:
 *   loss[i] = (1/count_i) sum_t (log sum_c exp Z[t][c] - Z[t][y_t])
 *                                          (DEVICE float [n]; 0 if count_i = 0)
 *   dZ[t][c] = (scale/count_i) (softmax(Z[t])_c - [c = y_t])
 * dZ (DEVICE, of dtype, row stride ld_dZ) may be NULL (no gradient) or Z
 * itself; it must not overlap Z otherwise.  Sums are held in fp32, a worker's
 * over its rows in fp64 in a fixed order.  Logits of -infinity, and those whose
 * probability is below 2^-126 of the row's largest, have probability 0; a row
 * with a NaN, a +infinity or only -infinities, and a row whose label is >= C,
 * give a NaN loss and a NaN gradient row.  scale must be finite.  n in [1, DBW_MAX_N], C in [1, 2^24], T below 2^31.  workspace
 * (DEVICE, 16-byte aligned, at least dbw_token_workspace bytes): as for
 * dbw_group_product. */
int64_t dbw_token_workspace(int32_t n, int64_t T);
dbw_status dbw_token_loss(int32_t n, int64_t T, int32_t C, int32_t dtype, const int32_t* offsets, const void* Z,
                          int64_t ld_Z, const int32_t* y, double scale, void* dZ, int64_t ld_dZ, float* loss,
                          void* workspace, int64_t workspace_bytes, void* stream);

/* AdamW over many tensors at once (the server's update of such a model).  One
 * step over all tensors, with t the number of steps made, this one included:
 *   norm = |grad_scale| sqrt(sum g^2) over all tensors,
 *   f    = grad_scale, times max_norm / norm where 0 < max_norm < norm,
 *   m <- beta1 m + (1 - beta1) f g,     v <- beta2 v + (1 - beta2) (f g)^2,
 *   w <- (1 - lr decay) w - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 * with a tensor's lr = hyper.lr * lr_scale and decay = weight_decay.  With
 * max_norm > 0, a norm that is not finite leaves everything as it was, t
 * included.  w is fp32; w_low (nullable) gets a copy rounded to low_dtype.
 *
 * state_bits = 32: m and v are float [count].  state_bits = 8: m holds m, and
 * v holds r = sqrt(v), as e4m3 codes (uint8 [count]) times a power of two for
 * each 256 values from the tensor's start, m_scale and v_scale (uint8
 * [ceil(count/256)], the biased exponent e of 2^(e-127)).  The scale puts the
 * largest finite magnitude of the 256, or 2^-118 if that is more, into (224,
 * 448].  A value between two codes takes the upper with the probability of its
 * place between them, by 16 bits of a mix of seed, t, tensor and index (see
 * dbw_adamw_bits), so that m and r keep their mean although a step's change
 * is far below a code; an r above 0 never becomes 0 (m/r stays bounded).
 * Values that are not finite become NaN codes.  The update itself uses m and
 * v before they are rounded. */
typedef struct {
  float* w;         /* DEVICE [count]                                        */
  const void* g;    /* DEVICE [count] of g_dtype                             */
  void *m, *v;      /* DEVICE [count]                                        */
  uint8_t *m_scale, *v_scale; /* DEVICE; NULL with 32-bit states             */
  void* w_low;      /* DEVICE [count] of low_dtype, or NULL                  */
  int64_t count;    /* >= 0; of all tensors together at most 2^36              */
  double lr_scale, weight_decay; /* finite, >= 0                             */
} dbw_adamw_tensor;
typedef struct {
  int32_t state_bits; /* 8 or 32                                             */
  int32_t g_dtype;    /* dbw_dtype of every g                                */
  int32_t low_dtype;  /* DBW_BF16 or DBW_F16, of every w_low                 */
  int32_t tensors;    /* in [1, 65536]                                       */
  int64_t t;          /* steps made so far, >= 0                             */
} dbw_adamw_config;
typedef struct {
  double lr, beta1, beta2, eps; /* lr >= 0, betas in [0, 1), eps >= 1e-30    */
  double grad_scale;            /* finite                                    */
  double max_norm;              /* 0: no clipping                            */
  uint32_t seed;
} dbw_adamw_hyper;
typedef struct dbw_adamw dbw_adamw;

/* A plan for these tensors on the current device: their addresses and t are
 * kept on the device until dbw_adamw_destroy.  An array that a step writes
 * (all but g) must overlap no other of the plan (DBW_EINVAL); two tensors may
 * read the same g.  Each pointer is aligned to its elements. */
dbw_status dbw_adamw_create(const dbw_adamw_config* cfg, const dbw_adamw_tensor* tensors, dbw_adamw** out);
void dbw_adamw_destroy(dbw_adamw* opt);

/* One step on `stream` of the plan's device (allocates nothing; t lives on
 * the device, so a captured step advances it at every replay).  norm, if not
 * NULL, is DEVICE float [1] and gets the norm before clipping (infinite where
 * fp32 cannot hold it: the step itself takes it in fp64).  Steps of one
 * plan must not run at the same time. */
dbw_status dbw_adamw_step(dbw_adamw* opt, const dbw_adamw_hyper* hyper, float* norm, void* stream);

/* t of a plan (checkpoint and resume; both wait for the plan's device). */
dbw_status dbw_adamw_export(dbw_adamw* opt, int64_t* t);
dbw_status dbw_adamw_import(dbw_adamw* opt, int64_t t);

/* AdamW as the server's update of dbw_step: from now on, and until another
 * call, each dbw_step on ctx ends with one step of opt (with hyper, copied) on
 * the context's stream instead of w <- w - eta g_t; opt NULL brings that back.
 * The gradients of opt's tensors must lie in the context's g_t
 * (dbw_step_outputs, a buffer that stays where it is), each at the place that
 * its w has in the w passed to dbw_step (DBW_EINVAL there otherwise); what no
 * tensor covers is not updated.  opt must be on the context's device and
 * outlive this use.  The estimator's formulas keep cfg.eta. */
dbw_status dbw_set_adamw(dbw_ctx* ctx, dbw_adamw* opt, const dbw_adamw_hyper* hyper);

/* The 32 random bits of value `index` of tensor `tensor` at step t (HOST; the
 * low 16 round m, the high 16 round r).  With mix(x): x ^= x >> 16, x *=
 * 0x9E3779B1, x ^= x >> 15, x *= 0xB7E15163, x ^= x >> 16 in 32 bits, they are
 * mix(lo * 0x6A09E667 + hi * 0xBB67AE85 + mix(mix(mix(seed) + t) + tensor))
 * for the halves lo and hi of index. */
uint32_t dbw_adamw_bits(uint32_t seed, int64_t t, int32_t tensor, int64_t index);

/* ---------------------------------------------------------------------------
 * A transformer block in training, beside the products, the loss and the
 * update above: attention, layer norm, the products with what surrounds them,
 * and dropout.  The rules above hold here too: no context, a stream, device
 * offsets of n ragged groups (the workers' rows; for attention the sequences),
 * nothing allocated, capturable; rows of no group are not read, and left as
 * they were in outputs.  Row strides are below 2^32, or what is said below
 * (DBW_EUNSUPPORTED above).  Outputs must not overlap inputs or each other, but for
 * what is said below (DBW_EINVAL where one is the other).  Vectors of weights
 * (gamma, beta, bias) are fp32, as AdamW keeps them, and so are their
 * gradients, one row for each worker: with the row stride P they lie in the
 * worker gradients G [n][P].  NaN and infinities of one group's rows never
 * reach another's. */

/* Layer norm: with the mean and variance (of all d values) of row t,
 *   H[t] = (X[t] - mean) / sqrt(var + eps),   Y[t] = H[t] gamma + beta.
 * X and Y are DEVICE [T][d] of dtype (row strides ld_X, ld_Y, in elements),
 * gamma and beta DEVICE float [d] (beta may be NULL: 0).  Statistics are formed
 * in fp32, the variance from differences to the mean: their squares' sum has to
 * be finite there (values below 2^56 in size always have that).  n in [1, DBW_MAX_N], d
 * in [1, 16384] (DBW_EUNSUPPORTED above), T below 2^31, eps in [1e-30, 1e30]. */
dbw_status dbw_layer_norm(int32_t n, int64_t T, int32_t d, int32_t dtype, const int32_t* offsets, const void* X,
                          int64_t ld_X, const float* gamma, const float* beta, double eps, void* Y, int64_t ld_Y,
                          void* stream);

/* Its gradients, from the same X (the statistics are formed again):
 *   dX[t] = (dH - mean(dH) - H mean(dH H)) / sqrt(var + eps),  dH = dY[t] gamma
 *   dgamma_i = sum over the rows t of group i of dY[t] H[t],  dbeta_i = sum dY[t]
 * dX is DEVICE [T][d] of dtype, dgamma and dbeta DEVICE float [n][d] (row
 * strides ld_dgamma, ld_dbeta; zero for an empty group; dbeta may be NULL).
 * The sums are taken in a fixed order.  workspace: as for dbw_group_product, at
 * least dbw_layer_norm_workspace bytes (-1 for arguments out of range). */
int64_t dbw_layer_norm_workspace(int32_t n, int64_t T, int32_t d);
dbw_status dbw_layer_norm_grad(int32_t n, int64_t T, int32_t d, int32_t dtype, const int32_t* offsets, const void* dY,
                               int64_t ld_dY, const void* X, int64_t ld_X, const float* gamma, double eps, void* dX,
                               int64_t ld_dX, float* dgamma, int64_t ld_dgamma, float* dbeta, int64_t ld_dbeta,
                               void* workspace, int64_t workspace_bytes, void* stream);

/* A product with bias, activation and residual:
 *   Z[t] = X[t] W_i + b_i,   Y[t] = act(Z[t]) + R[t]
 * for the rows t of group i; the FORWARD form of dbw_group_product, whose
 * shape, workspace and rules it has.  act(z) = z, max(z, 0), z / (1 + exp(-2 (a
 * z + b z^3))) with a = sqrt(2/pi), b = 0.044715 a (the tanh form of GELU), or z
 * / (1 + exp(-z)).  Z and Y are rounded once each, from the fp32 sum. */
typedef enum { DBW_ACT_NONE = 0, DBW_ACT_RELU = 1, DBW_ACT_GELU = 2, DBW_ACT_SILU = 3 } dbw_activation;
typedef struct {
  int32_t activation;   /* dbw_activation                                    */
  const float* bias;    /* DEVICE [C] of group i at bias + i st_bias, or NULL */
  int64_t st_bias;      /* >= C, or 0: the same for all groups, as it has to be
                           where the groups share W                          */
  const void* residual; /* DEVICE [T][C] of out_dtype, or NULL; may be Y     */
  int64_t ld_residual;  /* row stride, below 2^21; that of Y where it is Y   */
  void* pre;            /* DEVICE [T][C] of dtype: gets Z (for
                           dbw_linear_grad), or NULL                         */
  int64_t ld_pre;       /* row stride, below 2^21                            */
} dbw_linear_epilogue;
dbw_status dbw_group_linear(const dbw_group_shape* shape, const dbw_linear_epilogue* epilogue, const int32_t* offsets,
                            const void* X, const void* W, void* Y, void* workspace, int64_t workspace_bytes,
                            void* stream);

/* The way back to Z and the bias:
 *   dZ[t] = dY[t] act'(Z[t]),   dbias_i = sum over the rows t of group i of dZ[t]
 * (from there dbw_group_product: INPUT_GRAD and WEIGHT_GRAD of dZ; the
 * gradient to R is dY).  dY, Z and dZ are DEVICE [T][C] of dtype (fp32, bf16
 * or fp16); Z may be NULL with DBW_ACT_NONE, and dZ too (then only dbias is
 * formed).  dbias is DEVICE float [n][C], row stride ld_dbias, zero for an
 * empty group, a sum in a fixed order of the values before they are rounded;
 * NULL: not formed.  act'(0) of RELU is 0.  C in [1, 2^20].  workspace: at
 * least dbw_linear_grad_workspace bytes. */
int64_t dbw_linear_grad_workspace(int32_t n, int64_t T, int32_t C);
dbw_status dbw_linear_grad(int32_t n, int64_t T, int32_t C, int32_t dtype, int32_t activation, const int32_t* offsets,
                           const void* dY, int64_t ld_dY, const void* Z, int64_t ld_Z, void* dZ, int64_t ld_dZ,
                           float* dbias, int64_t ld_dbias, void* workspace, int64_t workspace_bytes, void* stream);

/* Causal attention over packed sequences: group i is a sequence, and for its
 * rows t and each of `heads` heads, whose keys and values are those of head
 * floor(head kv_heads / heads),
 *   S[t][s] = scale Q[t] . K[s]  for the rows s <= t of t's sequence,
 *   lse[t] = log sum_s exp S[t][s],   O[t] = sum_s exp(S[t][s] - lse[t]) V[s].
 * Products take bf16 or fp16 and sum in fp32; the exponentials are rounded to
 * dtype for the second product, and summed unrounded.  Arrays are DEVICE
 * [T][heads or kv_heads][D] of dtype, the D values contiguous; lse is DEVICE
 * float [heads][T], or NULL.  Q . K and S have to be finite in fp32, and may be
 * of any size there; a weight is off by the factor exp(error of S), S being a
 * sum of D products in fp32.  NaN and infinities of a row may reach all rows
 * of its sequence. */
typedef struct {
  void* data;             /* 16-byte aligned                                 */
  int64_t token, head;    /* elements from a token, or a head, to the next:
                             multiples of 8, token below 2^21, head below 2^40;
                             not below 0, and outputs' rows apart            */
} dbw_heads;
typedef struct {
  int32_t dtype;           /* DBW_BF16 or DBW_F16                            */
  int32_t n;               /* sequences, in [1, 65536]                       */
  int32_t heads, kv_heads; /* kv_heads divides heads; heads at most 1024     */
  int32_t D;               /* a multiple of 8, in [8, 128]                   */
  int64_t T;               /* rows, in [0, 2^31); (floor(T / 64) + n) heads
                              below 2^23 (DBW_EUNSUPPORTED)                  */
  double scale;            /* in [1e-20, 1e20]                               */
} dbw_attention_shape;
dbw_status dbw_attention(const dbw_attention_shape* shape, const int32_t* offsets, const dbw_heads* Q,
                         const dbw_heads* K, const dbw_heads* V, const dbw_heads* O, float* lse, void* stream);

/* Its gradients, from O and lse of the call above:
 *   P[t][s] = exp(S[t][s] - lse[t]),   dV[s] = sum_t P[t][s] dO[t],
 *   dS[t][s] = P[t][s] (dO[t] . V[s] - dO[t] . O[t]),
 *   dQ[t] = scale sum_s dS[t][s] K[s],   dK[s] = scale sum_t dS[t][s] Q[t]
 * with dK and dV summed over the heads that share them, in a fixed order.  P
 * and dS are rounded to dtype for the products.  Where |lse| is above 709 for a
 * row, its 128 take maximum and sum from Q and K again, as lse does not hold
 * exp(S - lse) to its last digits there.  workspace: at least
 * dbw_attention_workspace bytes (-1 for a shape out of range). */
int64_t dbw_attention_workspace(const dbw_attention_shape* shape);
dbw_status dbw_attention_grad(const dbw_attention_shape* shape, const int32_t* offsets, const dbw_heads* dO,
                              const dbw_heads* Q, const dbw_heads* K, const dbw_heads* V, const dbw_heads* O,
                              const float* lse, const dbw_heads* dQ, const dbw_heads* dK, const dbw_heads* dV,
                              void* workspace, int64_t workspace_bytes, void* stream);

/* Dropout, with a mask that is never stored:
 *   Y[t][c] = R[t][c] + (u[t][c] >= q ? X[t][c] * 65536 / (65536 - q) : 0)
 * with q = round(65536 p), p in [0, 1] (q = 65536: Y = R), and u the 16 random
 * bits of a value: those at 16 (c mod 8) of the 128 bits of Philox4x32-10
 * (Salmon, Moraes, Dror and Shaw, 2011), with the low half of each word before
 * its high half, counter (floor(c/8), t, low and high half of *step), key (low
 * and high half of seed); see dbw_dropout_bits.  The gradient to X is the same
 * call on dY, without R.  X, Y and R (may be NULL: 0) are DEVICE [T][d] of
 * dtype; Y may be X or R, with its row stride.  step is DEVICE int64 [1] (NULL:
 * 0), so that a captured call draws anew at each replay.  d in [1, 2^20]. */
dbw_status dbw_dropout(int32_t n, int64_t T, int32_t d, int32_t dtype, const int32_t* offsets, const void* X,
                       int64_t ld_X, double p, uint64_t seed, const int64_t* step, const void* R, int64_t ld_R,
                       void* Y, int64_t ld_Y, void* stream);

/* The 16 bits u of value [t][c] (HOST). */
uint32_t dbw_dropout_bits(uint64_t seed, int64_t step, int64_t t, int32_t c);

#ifdef __cplusplus
}
#endif

#endif /* DBW_H */
