/*
 * hier_avg.h - C ABI of the Hier-AVG data-parallel hot path on one GPU.
 *
 * Hier-AVG is Algorithm 1 (Sec. 3.1) of Zhou & Cong, "A Distributed Hierarchical
 * Averaging SGD Algorithm: Trading Local Reductions for Global Reductions".  All
 * P learners live on one GPU as rows of a learner-indexed fp32 parameter matrix
 * [P, ld]; the paper's local and global reductions become in-memory segmented and
 * full means over the learner axis.
 *
 * Conventions shared by every call
 *   - Every pointer argument named *_dev is a device pointer on the current CUDA
 *     device; *_host pointers are host memory.  Nothing is freed by the library
 *     that the caller passed in; the caller keeps ownership of all buffers and
 *     must keep them alive while work that uses them is in flight.
 *   - All compute calls are asynchronous on the CUDA stream given to them (or
 *     bound to the handle); a NULL stream is the legacy default stream.  Only
 *     hier_avg_losses, hier_avg_check, hier_avg_operator_check, hier_avg_round_host
 *     and the profile read synchronise.
 *   - No call changes the calling thread's current CUDA device: a call that runs
 *     work on the handle's device makes it current and restores the caller's.
 *   - Every call returns HA_OK (0) or a negative status; nothing aborts.
 *     hier_avg_strerror() names a status, hier_avg_last_error() gives the
 *     message of the handle's last failure.
 *   - K2 counts LOCAL AVERAGES per global average (the paper's beta, Sec. 3.1);
 *     the paper's global interval in local steps is K1 * K2.
 */
#ifndef HIER_AVG_H
#define HIER_AVG_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define HA_OK            0
#define HA_EINVAL       (-1)  /* an argument is out of range or inconsistent        */
#define HA_ENOMEM       (-2)  /* a caller-provided buffer is too small              */
#define HA_ECUDA        (-3)  /* a CUDA runtime or driver call failed               */
#define HA_ESTATE       (-4)  /* call out of order (e.g. a step before bind)        */
#define HA_ETIMEOUT     (-5)  /* a bounded device-side wait expired; see check      */
#define HA_EUNSUPPORTED (-6)  /* valid request the library does not implement       */

#define HA_PREC_FP32 0        /* every product in fp32 on CUDA cores                */
#define HA_PREC_BF16 1        /* bf16 GEMM operands, fp32 accumulate, fp32 master   */

/* ---------------------------------------------------------------------------
 * Stateless averaging on a caller's learner-indexed buffer.
 *
 * w_dev: P rows of D fp32 values, row j starting at w_dev + j * ld (ld >= D).
 * The mean of n rows is their sum in the canonical adjacent-pair tree order
 * (levels h = 1, 2, 4, ...: v[i] += v[i+h] for i = 0, 2h, ..., an unpaired
 * element carried up), then one correctly rounded fp32 division by n; no FMA,
 * no flush of subnormals.  The result is therefore bit-reproducible.
 * Errors: HA_EINVAL if P < 1, D < 0, ld < D, S < 1, P % S != 0 or w_dev is NULL
 * with D > 0; HA_ECUDA if the launch fails.  D = 0 is a no-op.
 * ------------------------------------------------------------------------- */

/* Local average, Algorithm 1 (Sec. 3.1) "locally average and synchronize":
 * every row of cluster g (rows [g*S, (g+1)*S)) is replaced by the cluster mean. */
int hier_avg_local_average_buffer(float* w_dev, int64_t P, int64_t S, int64_t D,
                                  int64_t ld, void* stream);

/* Global average, Algorithm 1 (Sec. 3.1) "globally average and synchronize"
 * together with the synchronisation at the top of the next round: every row is
 * replaced by the mean over all P rows. */
int hier_avg_global_average_buffer(float* w_dev, int64_t P, int64_t D, int64_t ld,
                                   void* stream);

/* The last local average of a round followed by the global average (Algorithm 1,
 * end of the b-loop then the global step), in one pass over memory.  Bit-identical
 * to hier_avg_local_average_buffer followed by hier_avg_global_average_buffer. */
int hier_avg_local_global_average_buffer(float* w_dev, int64_t P, int64_t S, int64_t D,
                                         int64_t ld, void* stream);

/* ---------------------------------------------------------------------------
 * Handle API: P learners of a ReLU MLP d_0 -> d_1 -> ... -> d_L trained with
 * mean softmax cross-entropy (the learner objective; Algorithm 1 leaves F open).
 * ------------------------------------------------------------------------- */
typedef struct hier_avg hier_avg;

/* Validate a configuration and create a handle (host memory only, no GPU work).
 *   P, S, K1, K2, lr, B : Sec. 2 notation (K2 = local averages per round), S | P
 *   dims[0..n_dims-1]   : d_0 .. d_L, n_dims = L + 1 >= 2, every d >= 1
 *   precision           : HA_PREC_FP32 or HA_PREC_BF16
 * Errors: HA_EINVAL for P, S, K1, K2, B < 1, P % S != 0, non-finite lr, bad dims or
 * precision; HA_EUNSUPPORTED for a shape the kernels do not cover (BF16: B > 64 or
 * an input width d_0 .. d_{L-1} not a multiple of 8; either: P > 65535). */
int hier_avg_create(int P, int S, int K1, int K2, float lr, int B, const int* dims,
                    int n_dims, int precision, hier_avg** out);

/* Free the handle (never the caller's buffers).  NULL is a no-op. */
void hier_avg_destroy(hier_avg* h);

/* Parameter layout of one learner row.  *D = parameters per learner,
 * *ld = padded row length in floats (multiple of 64; padding stays zero).
 * offsets (2 * L entries, may be NULL): offsets[2l] = start of W_{l+1}
 * ([d_{l+1}, d_l] row-major), offsets[2l+1] = start of b_{l+1} ([d_{l+1}]). */
int hier_avg_param_layout(const hier_avg* h, int64_t* D, int64_t* ld, int64_t* offsets);

/* Bytes of device workspace hier_avg_bind needs: a step's scratch and, for the bf16
 * path with S > 1, the cluster means [P / S, ld] fp32 that hier_avg_round's local
 * averages write. */
int hier_avg_workspace_bytes(const hier_avg* h, int64_t* bytes);

/* Attach device memory (all borrowed, caller-owned) and the stream:
 *   params_dev    [P, ld] fp32, the learner replicas (initialised by the caller,
 *                 e.g. one w0 copied to every row: Algorithm 1 starts from one
 *                 global parameter)
 *   workspace_dev >= hier_avg_workspace_bytes bytes, 256-byte aligned; zeroed here
 *   X_dev         [P, N, d_0] per-learner samples, bf16 for HA_PREC_BF16, fp32
 *                 for HA_PREC_FP32; y_dev [P, N] int32 labels in [0, d_L)
 * Builds the TMA descriptors.  Resets the step counter to 0.
 * Errors: HA_EINVAL (NULL pointer, N < 1, misaligned params or workspace),
 * HA_ENOMEM (workspace too small), HA_ECUDA. */
int hier_avg_bind(hier_avg* h, float* params_dev, void* workspace_dev,
                  int64_t workspace_bytes, const void* X_dev, const int32_t* y_dev,
                  int64_t N, void* stream);

/* One local SGD step of every learner, Algorithm 1 inner loop (Sec. 3.1):
 * w_j <- w_j - (lr / B) * sum_s grad f(w_j; xi_{j,s}).  Learner j at step t uses
 * rows (t*B + s) mod N of its own data.  Then t <- t + 1.  HA_ESTATE before bind. */
int hier_avg_step(hier_avg* h);

/* Local average of the bound parameters (see hier_avg_local_average_buffer). */
int hier_avg_local_average(hier_avg* h);

/* Global average of the bound parameters (see hier_avg_global_average_buffer). */
int hier_avg_global_average(hier_avg* h);

/* One global round of Algorithm 1: K2 x (K1 x step, local average), then the
 * global average; the last local average is fused with the global one
 * (bit-identical to doing them in turn).  The other local averages write each
 * cluster's mean once, into the workspace, and the step that follows reads every
 * learner's parameters from its cluster's mean (forwarding groups of a cluster's
 * learners with one product per weight tile) and writes the learner's row.  With S
 * even (bf16 path), the step before each average stores, instead of every learner's
 * updated weights, the sums of pairs or quads of a cluster's learners (the first
 * levels of the averaging tree) in the first learner row of each pair or quad, and the
 * average finishes the tree from them.  So within a round the rows of params_dev are
 * scratch; the values every step and average computes are those of the literal
 * sequence, and when the round returns every row holds its learner's parameters.
 * Within the round, a step whose successor starts no local block and reads a
 * contiguous batch also computes that successor's first-layer output from the weights
 * it has just updated (bf16 path, two or more layers), so W_1 is read once per step;
 * the results are those of calling hier_avg_step, hier_avg_local_average and
 * hier_avg_global_average in turn, bit for bit. */
int hier_avg_round(hier_avg* h);

/* Global averaging interval in local steps: hier_avg_round then runs `steps` local
 * steps, a local average after every K1-th of them, and the global average after the
 * last, preceded by a local average exactly when K1 divides `steps`.  Sec. 3.1 takes
 * the interval K1 * beta with beta an integer for the analysis and leaves it free in
 * practice (Sec. 4's ImageNet run: K1 = 20, 43 steps).  0 restores K1 * K2 (the
 * default).  HA_EINVAL for steps < 0 or a NULL handle. */
int hier_avg_set_global_steps(hier_avg* h, int steps);

/* Step size of the following local steps (the gamma_n of round n; Theorem 3.3's
 * diminishing schedules set it between rounds).  HA_EINVAL if lr is not finite. */
int hier_avg_set_lr(hier_avg* h, float lr);

/* Mini-batch size of the following local steps (the B_n of round n; Theorem 3.3's
 * growing batches), 1 <= B <= the B given at create (which sizes the buffers).  Each
 * learner reads its data sequentially: a step's batch starts where the previous one
 * ended, at row (rows read so far) mod N, which is t * B for a constant B.
 * HA_EINVAL outside that range; HA_ECUDA if clearing device buffers fails. */
int hier_avg_set_batch(hier_avg* h, int B);

/* One round end to end from host memory: copies the rows of X_host [P, N, d_0] that
 * this round reads, and all of y_host [P, N] (P * N * 4 bytes, one copy), into the
 * bound device data set (pinned host memory recommended), runs hier_avg_round, and
 * copies the per-learner loss of the round's last step into loss_host [P].  The rows
 * of X go in chunks of steps that double in length, on a stream of the library's own,
 * issued between the kernel launches, and overlap the kernels: a step waits only for
 * the chunk holding the rows it reads (bf16 path; the fp32 path copies the round's
 * rows first).  A chunk whose rows span at least 512 KB per learner is one copy per
 * learner when a learner's parameter row holds at least 4 Mi values, otherwise a
 * single pitched copy for all learners.  Synchronises. */
int hier_avg_round_host(hier_avg* h, const void* X_host, const int32_t* y_host,
                        float* loss_host);

/* One local step, exactly as hier_avg_step, for callers that cannot allocate
 * device memory (no cudaMalloc in their environment, an allocator they do not
 * own, or a binding that only passes existing buffers).  The paper has no
 * counterpart: this is a property of the library, not of the method.
 * The caller passes the inputs and outputs (params_dev [P, ld] updated in place,
 * X_dev, y_dev, N as for hier_avg_bind); the step's scratch lives in one 32 MiB
 * array that the library holds in every GPU's memory until the process exits.
 * The call binds the handle to these buffers and to that array, clears the part
 * of the array the step uses, takes the step at the handle's counter t and
 * advances t.  It calls no device allocator.
 *   - The first call in each CUDA context of a device (so once per device, and
 *     again after a device reset) looks up the array's device address; make that
 *     first call before any stream capture on that device.
 *   - Every call, from any handle, shares the one array and leaves its contents
 *     behind; calls whose work overlaps on the GPU (other streams, other
 *     threads) race on it.  After a call, later hier_avg_step / round calls of
 *     the same handle also use the array until hier_avg_bind is called again.
 * Errors: HA_ENOMEM (with a message naming both sizes) when one step of the
 * configuration needs more than 32 MiB of scratch (hier_avg_workspace_bytes less
 * the cluster means, which only rounds use; a round of a handle bound this way
 * averages in place), HA_EINVAL for NULL or misaligned buffers or N < 1, HA_ECUDA. */
int hier_avg_step_static(hier_avg* h, float* params_dev, const void* X_dev,
                         const int32_t* y_dev, int64_t N, void* stream);

/* Step counter t (local SGD steps taken); setting it resumes a run whose
 * parameters were saved: it also sets the rows read so far to t * B (the current
 * batch size), which is where a run with a constant batch size stands. */
int hier_avg_get_step(const hier_avg* h, int64_t* t);
int hier_avg_set_step(hier_avg* h, int64_t t);

/* Per-learner mean cross-entropy of the last step's mini-batch -> loss_host [P].
 * Synchronises the bound stream. */
int hier_avg_losses(hier_avg* h, float* loss_host);

/* Synchronise the bound stream and report a device-side failure:
 * HA_ETIMEOUT if a bounded wait inside a kernel expired (that kernel stopped
 * early and its outputs are invalid), HA_ECUDA on an asynchronous CUDA error. */
int hier_avg_check(hier_avg* h);

/* Failure-detection self-test (the paper has no counterpart: this checks the
 * library's own failure detection).  Launches one kernel on the bound stream that
 * runs the library's two kinds of bounded device wait -- an acquire spin on a global
 * flag and an mbarrier phase wait, the waits that order split-K reductions and the
 * TMA / tensor-core pipelines -- on conditions nothing will satisfy, each with a limit
 * of limit_us microseconds at the device's peak SM clock (longer at a lower clock).
 * Both expire; the kernel records the timeout in the handle's error word and returns
 * with nothing in flight, so the CUDA context stays usable.  The next hier_avg_check
 * returns HA_ETIMEOUT and clears the word; later calls work as before.
 * Errors: HA_ESTATE before bind, HA_EINVAL for limit_us outside [1, 1e7], HA_ECUDA. */
int hier_avg_wait_selftest(hier_avg* h, int64_t limit_us);

/* Kernel timing with CUDA events recorded on the bound stream around every
 * launch of the handle.  enable = 1 starts (and clears) it, 0 stops it. */
#define HA_KERNEL_GATHER        0   /* mini-batch fetch (+ transpose)        */
#define HA_KERNEL_FORWARD       1   /* per-layer forward GEMM + epilogue     */
#define HA_KERNEL_XENT          2   /* softmax cross-entropy gradient        */
#define HA_KERNEL_BACKWARD      3   /* fused dX + dW + SGD update            */
#define HA_KERNEL_LOCAL_AVG     4
#define HA_KERNEL_GLOBAL_AVG    5   /* fused last local + global average     */
#define HA_KERNEL_HEAD          6   /* fused last layer (<= 16 classes)      */
#define HA_KERNEL_UPDATE_FORWARD 7  /* first-layer update + next forward     */
#define HA_KERNEL_KINDS         8
int hier_avg_profile(hier_avg* h, int enable);

/* The same for a subset: kinds is a bitmask of (1 << HA_KERNEL_*); 0 stops.
 * Each timed launch costs two event records that separate it from its
 * neighbours on the stream, so a throughput measurement times only the kinds it
 * reports.  HA_EINVAL for bits beyond HA_KERNEL_KINDS. */
int hier_avg_profile_kinds(hier_avg* h, unsigned kinds);

/* Kernels this handle has launched since it was created (every launch of the step,
 * averaging and round calls, one per kernel).  HA_EINVAL for NULL arguments. */
int hier_avg_launches(const hier_avg* h, int64_t* launches);

/* Time only every n-th launch of each enabled kind (n >= 1, default 1; counted from
 * the last hier_avg_profile / hier_avg_profile_kinds), so that a throughput
 * measurement perturbs few launches.  hier_avg_profile_read then reports the
 * sampled launches.  HA_EINVAL for n < 1. */
int hier_avg_profile_every(hier_avg* h, int every);

/* Synchronise and read kind's totals since profiling was enabled: summed event
 * time in ms, number of launches, the algorithmic bytes moved by them (fp32 master
 * read and written, activations read and written once) and their algorithmic flops
 * (2 per multiply-add of the step's products: forward, dW and dX of every learner;
 * P * ld additions per average).  Any output pointer may be NULL. */
int hier_avg_profile_read(hier_avg* h, int kind, double* total_ms, int64_t* launches,
                          double* bytes, double* flops);

/* ---------------------------------------------------------------------------
 * Operators for models whose groups of rows have weights of their own (experts, or
 * learners with batches of different sizes), for their loss over many classes, and
 * for steps other than plain SGD.  Stateless but for the AdamW plan.  They run on the
 * current device, asynchronously on `stream`, and allocate nothing.  All sums are held
 * in fp32.
 * ------------------------------------------------------------------------- */
#define HA_TYPE_FP32 0
#define HA_TYPE_BF16 1
#define HA_TYPE_FP16 2

/* Grouped products.  Rows [offsets[g], offsets[g+1]) of x (and dy) belong to group g,
 * which has the weights W_g [outer, inner]; offsets_dev [groups + 1] int32 stays on the
 * device and is not read by the host.  Groups may be empty and of any size; offsets are
 * clamped to [0, rows], and one that goes back leaves its group empty.
 *   hier_avg_grouped_product     y[t]  = act(W_g x[t] + b_g)
 *   hier_avg_grouped_product_dx  dx[t] = W_g^T dy[t], zero where h[t] <= 0 (h_dev != NULL)
 *   hier_avg_grouped_product_dw  dW_g  = sum over the group's t of dy[t] x[t]^T, and with
 *                                db_dev db_g = sum of dy[t]; zero for an empty group
 * Rows of y and dx that belong to no group are set to zero; where offsets go back, a row of y or
 * dx that lies in two groups is the first one's (dW and db count it in both).
 *   type          HA_TYPE_BF16 or HA_TYPE_FP16, of x, w, dy and h; products are exact and
 *                 summed in fp32
 *   y_type, ...   the inputs' type (rounded once) or HA_TYPE_FP32
 *   *_ld          elements between rows; w_gs, dw_gs: between groups; unit stride inside
 *                 rows.  bias_dev [groups, outer] and db_dev fp32, rows bias_ld / db_ld apart
 *   relu          1: act(v) = max(v, 0), 0: act(v) = v
 *   workspace_dev 16-byte aligned, of the bytes that hier_avg_grouped_product_workspace says
 *                 (0 for operands whose address and strides are multiples of 16 bytes and
 *                 whose groups and rows do not overlap;
 *                 others are first copied there, and a weights' gradient of few tiles over
 *                 many rows has its parts there before they are added)
 * Errors: HA_EINVAL for sizes, types, strides or pointers out of range, HA_ENOMEM for a
 * workspace that is too small, HA_EUNSUPPORTED for more than 1024 groups or 2^31 tiles,
 * HA_ECUDA.  rows = 0 is valid (dW is then zero). */
#define HA_GROUPED_FORWARD 0
#define HA_GROUPED_DX 1
#define HA_GROUPED_DW 2
/* a: x (forward) or dy; b: w (forward, dx) or x (dw; b_gs is not read). */
int hier_avg_grouped_product_workspace(int op, const void* a_dev, int64_t a_ld, const void* b_dev,
                                       int64_t b_ld, int64_t b_gs, int groups, int64_t rows,
                                       int inner, int outer, int64_t* bytes);
int hier_avg_grouped_product(const void* x_dev, int64_t x_ld, const void* w_dev, int64_t w_ld,
                             int64_t w_gs, int type, const int32_t* offsets_dev, int groups,
                             int64_t rows, int inner, int outer, const float* bias_dev,
                             int64_t bias_ld, int relu, void* y_dev, int64_t y_ld, int y_type,
                             void* workspace_dev, int64_t workspace_bytes, void* stream);
int hier_avg_grouped_product_dx(const void* dy_dev, int64_t dy_ld, const void* w_dev, int64_t w_ld,
                                int64_t w_gs, int type, const int32_t* offsets_dev, int groups,
                                int64_t rows, int inner, int outer, const void* h_dev,
                                int64_t h_ld, void* dx_dev, int64_t dx_ld, int dx_type,
                                void* workspace_dev, int64_t workspace_bytes, void* stream);
int hier_avg_grouped_product_dw(const void* dy_dev, int64_t dy_ld, const void* x_dev, int64_t x_ld,
                                int type, const int32_t* offsets_dev, int groups, int64_t rows,
                                int inner, int outer, void* dw_dev, int64_t dw_ld, int64_t dw_gs,
                                int dw_type, float* db_dev, int64_t db_ld, void* workspace_dev,
                                int64_t workspace_bytes, void* stream);

/* Log probabilities of given classes.  With z_j = logits_j / temperature over the allowed
 * classes of a row:
 *   lse = log sum_j e^{z_j},  logp = z_target - lse,  entropy = -sum_j p_j log p_j,
 * and the `top` likeliest classes with their log probabilities, equal logits in the order
 * of their index.
 *   logits_dev  [rows, classes], rows ld apart, any HA_TYPE_*
 *   targets_dev [rows], int32 or int64 (target_bytes 4 or 8); below 0: logp is 0 and has no
 *               gradient; a target >= classes gives NaN
 *   allowed_dev NULL, or one byte a class, not 0 where it is allowed: [rows, classes] with
 *               rows allowed_ld apart, or [classes] for all rows with allowed_ld = 0
 *   temperature 2^-126 .. 1e27
 *   top         0 .. 32; top_logp_dev, top_index_dev [rows, top]
 * A logit at or below -1e30 counts as not allowed.  A row without an allowed class has
 * lse = logp = -inf and entropy 0; alternatives that do not exist have index -1 and
 * -inf.  A row with NaN or +inf among its allowed logits gives NaN (indices -1).
 * Errors: HA_EINVAL; HA_EUNSUPPORTED for top > 32 or more than 2^31 blocks; HA_ECUDA. */
int hier_avg_token_logprobs(const void* logits_dev, int type, int64_t rows, int64_t classes,
                            int64_t ld, const void* targets_dev, int target_bytes,
                            const uint8_t* allowed_dev, int64_t allowed_ld, float temperature,
                            int top, float* logp_dev, float* entropy_dev, float* lse_dev,
                            float* top_logp_dev, int32_t* top_index_dev, void* stream);
/* The gradient with respect to the logits, from the forward's lse and entropy and the
 * gradients dlogp_dev and dentropy_dev [rows] (dentropy_dev NULL: zero, and entropy_dev is
 * not read).  dlogits_dev has the logits' type and may be logits_dev itself (with the same
 * ld).  Zero where a class is not allowed, and in a row without an allowed class.  A target
 * >= classes, or a row whose lse is NaN, gives NaN (where allowed_dev does not say no).  The
 * probabilities are as exact as lse, which holds its value to 24 bits. */
int hier_avg_token_logprobs_backward(const void* logits_dev, int type, int64_t rows,
                                     int64_t classes, int64_t ld, const void* targets_dev,
                                     int target_bytes, const uint8_t* allowed_dev,
                                     int64_t allowed_ld, float temperature, const float* lse_dev,
                                     const float* entropy_dev, const float* dlogp_dev,
                                     const float* dentropy_dev, void* dlogits_dev,
                                     int64_t dlogits_ld, void* stream);

/* AdamW over many tensors in one launch:
 *   m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2
 *   p <- p (1 - lr decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32, g being the gradient times *grad_scale_dev (NULL: 1).
 * A plan is made once for a list of pieces (contiguous runs of fp32 parameters, in order of
 * their tensor): piece i is p_dev[i][0 .. n[i]), its 16-bit copy (copy_dev or an entry of it
 * may be NULL) and its gradient, which starts at element grad_offset[i] of tensor[i]'s
 * gradient; decay[i] is its weight decay.  The state arrays hold the pieces one after the
 * other, each from a multiple of 256 elements on (zeros between them).
 *   bits = 32   m_dev, v_dev: fp32 [elements]
 *   bits = 8    m_dev, v_dev: e4m3 [elements], m_scale_dev, root_scale_dev: fp32
 *               [elements / 256]; m = code * scale, and v_dev holds sqrt(v) in the same way,
 *               rounded up or down at random by `seed` and the element's place.  A block with
 *               a NaN or an infinity becomes NaN as a whole.
 * hier_avg_adamw_bind copies the plan to table_dev (16-byte aligned) and keeps the addresses.
 * t counts steps from 1.  Errors: HA_EINVAL (eps must be >= 2^-126, betas in [0, 1), a plan's
 * elements at most 2^37), HA_ENOMEM,
 * HA_ESTATE for a step before bind, HA_ECUDA. */
typedef struct hier_avg_adamw hier_avg_adamw;
int hier_avg_adamw_create(int bits, int n_tensors, int64_t n_pieces, const int* tensor,
                          float* const* p_dev, void* const* copy_dev, int copy_type,
                          const int64_t* n, const int64_t* grad_offset, const float* decay,
                          hier_avg_adamw** out);
void hier_avg_adamw_destroy(hier_avg_adamw* plan);
int hier_avg_adamw_sizes(const hier_avg_adamw* plan, int64_t* elements, int64_t* table_bytes);
int hier_avg_adamw_bind(hier_avg_adamw* plan, void* table_dev, int64_t table_bytes, void* m_dev,
                        void* v_dev, float* m_scale_dev, float* root_scale_dev, void* stream);
int hier_avg_adamw_step(hier_avg_adamw* plan, const void* const* grads_dev, int grad_type,
                        double lr, double beta1, double beta2, double eps, int64_t t,
                        const float* grad_scale_dev, uint32_t seed, void* stream);

/* Routing.  For each row of logits_dev [rows, experts] the k largest logits, from the largest down and equal ones by
 * index; a logit at or below -1e30 is masked.
 *   lse = log sum_i e^{z_i};  weight_j = e^{z_j} / (sum over the chosen of e^z), or e^{z_j - lse} (over_all)
 * Entries that do not exist have expert -1 and weight 0; a row with NaN or +inf has experts -1, and NaN weights and
 * lse; a row that is masked as a whole has lse -inf.
 * The entries (row, j) are then sorted by group, in their order within a group.  An entry's group is its expert, or,
 * with learners_dev [learners + 1] (rising int32 offsets on the device: learner p has the rows
 * learners[p] .. learners[p+1]), learner * experts + expert; rows of no learner have no group.
 *   expert_dev, weight_dev  [rows, k]
 *   offsets_dev             [groups + 1], as the grouped products read them
 *   place_dev               [rows, k] the entry's place among the sorted, -1: none
 *   source_dev              [rows * k] the entry row * k + j at each place, -1 behind the last group
 *   workspace_dev           16-byte aligned, of hier_avg_sort_workspace's bytes (0 for few rows)
 * hier_avg_sort_by_group sorts given groups group_dev [rows, per_row] (below 0 or >= groups: none).
 * hier_avg_route_backward takes dweight_dev [rows, k] to the logits' gradient: zero but for the chosen ones, or with
 * over_all for every expert (logits_dev and lse_dev are read only then; dlogits_dev may be logits_dev itself with the
 * same ld).  Rows whose weights are NaN give NaN.
 * Errors: HA_EINVAL; HA_EUNSUPPORTED for k or per_row > 32, more than 1024 experts or groups, or 2^31 entries;
 * HA_ENOMEM; HA_ECUDA. */
int hier_avg_sort_workspace(int64_t rows, int per_row, int groups, int64_t* bytes);
int hier_avg_route(const void* logits_dev, int type, int64_t rows, int experts, int64_t ld, int k, int over_all,
                   const int32_t* learners_dev, int learners, int32_t* expert_dev, float* weight_dev, float* lse_dev,
                   int32_t* offsets_dev, int32_t* place_dev, int32_t* source_dev, void* workspace_dev,
                   int64_t workspace_bytes, void* stream);
int hier_avg_sort_by_group(const int32_t* group_dev, int64_t rows, int per_row, int groups, int32_t* offsets_dev,
                           int32_t* place_dev, int32_t* source_dev, void* workspace_dev, int64_t workspace_bytes,
                           void* stream);
int hier_avg_route_backward(const float* dweight_dev, const void* logits_dev, int type, int64_t rows, int experts,
                            int64_t ld, int k, int over_all, const int32_t* expert_dev, const float* weight_dev,
                            const float* lse_dev, void* dlogits_dev, int64_t dlogits_ld, void* stream);

/* Rows to their groups and back, by the places of a sort: place_dev [rows, per_row], each place in
 * [0, rows * per_row) named once, others (-1) nowhere.  offsets_dev [groups + 1]: of it only the last is read,
 * behind which the sorted rows are set to zero.  (An entry is dropped by sorting again with its group below 0; where
 * only its place is overwritten, its sorted row is not written and stays in its group.)
 *   hier_avg_dispatch          xs[place[t, j]] = x[t]
 *   hier_avg_combine           out[t] = sum over j of weight[t, j] y[place[t, j]], in the order of j in fp32
 *                              (weight_dev NULL: 1 each, which is the gradient of dispatch); where there is no place,
 *                              weight[t, j] times 0, which is NaN where the weight is NaN or infinite
 *   hier_avg_combine_backward  dy[place[t, j]] = weight[t, j] dout[t],  dweight[t, j] = <dout[t], y[place[t, j]]>
 *                              (0 where there is no place)
 *   type                       any HA_TYPE_*, of x, xs, y and dy; out and dout: the same or HA_TYPE_FP32
 * Errors: HA_EINVAL, HA_EUNSUPPORTED for 2^31 entries or rows of more than 2^30 elements, HA_ECUDA. */
int hier_avg_dispatch(const void* x_dev, int type, int64_t rows, int width, int64_t x_ld, const int32_t* place_dev,
                      int per_row, const int32_t* offsets_dev, int groups, void* xs_dev, int64_t xs_ld, void* stream);
int hier_avg_combine(const void* y_dev, int type, int64_t rows, int width, int64_t y_ld, const int32_t* place_dev,
                     int per_row, const float* weight_dev, void* out_dev, int64_t out_ld, int out_type, void* stream);
int hier_avg_combine_backward(const void* dout_dev, int dout_type, int64_t dout_ld, const void* y_dev, int type,
                              int64_t rows, int width, int64_t y_ld, const int32_t* place_dev, int per_row,
                              const float* weight_dev, const int32_t* offsets_dev, int groups, void* dy_dev,
                              int64_t dy_ld, float* dweight_dev, void* stream);

/* The norm of all gradients together, sqrt(sum of their squares), and the factor that clips them: max_norm / norm
 * where norm > max_norm, else 1 (a NaN among them: norm NaN, factor 1).  Tensor i has n[i] contiguous elements of
 * types[i] at grads_dev[i].  learners > 1: every tensor's first dimension is the learner's (n[i] is a multiple of
 * learners), and norm_dev and scale_dev [learners] have one of each.  clip: the gradients are then multiplied by
 * their factor in place, each rounded once; they must not share memory.  scale_dev may be NULL without clip, and
 * max_norm is then not read.  Squares are summed so that neither their size nor their number is lost: in fp32 over at
 * most 32 KB, in 64 bits beyond, and in 64 bits at once where fp32's range does not hold them.
 * workspace_dev: 8-byte aligned, of hier_avg_grad_norm_workspace's bytes.
 * Errors: HA_EINVAL (gradients that share memory among them), HA_EUNSUPPORTED for more than 44800 tensors, 2^46
 * elements of one or 2^31 parts of 32 KB (2 KB of small tensors), HA_ENOMEM, HA_ECUDA. */
int hier_avg_grad_norm_workspace(int tensors, const int* types, const int64_t* n, int learners, int64_t* bytes);
int hier_avg_grad_norm(int tensors, void* const* grads_dev, const int* types, const int64_t* n, int learners,
                       double max_norm, int clip, float* norm_dev, float* scale_dev, void* workspace_dev,
                       int64_t workspace_bytes, void* stream);

/* Verification of drafted tokens.  A sequence has K = drafts drafts and K + 1 rows of logits; row i's probabilities
 * are p_i = softmax(logits_i / temperature) over the allowed classes, and draft i was drawn from probs_i.
 *   draft i is accepted while uniform_i * probs_i(draft_i) < p_i(draft_i) (probs_dev NULL: 1 for probs_i(draft_i));
 *   n, the accepted, is the first that is not, or the first draft below 0 (no draft), or K;
 *   the next token is argmax_j r_j / noise_j, the lowest index of equal ones: r = max(p_n - probs_n, 0) after a
 *   rejection (without probs: p_n without the draft; p_n where nothing is left), p_n otherwise.
 * With uniform numbers in [0, 1) and exponential noise the tokens are drawn as from the target itself; K = 0 draws
 * one token from p.  Decisions are those of exact arithmetic on the given numbers, unless the two sides of one are
 * within 2^-40 of each other.
 *   logits_dev   [sequences, K + 1, classes], sequences logits_seq and rows logits_row apart
 *   drafts_dev   [sequences, K] int32 or int64 (draft_bytes 4 or 8); a draft >= classes is rejected
 *   uniform_dev  [sequences, K];  noise_dev [sequences, classes], rows noise_ld apart, positive
 *   probs_dev    [sequences, K, classes] of any HA_TYPE_*, or NULL
 *   allowed_dev  NULL, or one byte a class, not 0 where it is allowed (strides 0: the same for all)
 *   tokens_dev   [sequences, K + 1]: the accepted drafts, the next token, then -1
 *   logp_dev     [sequences, K + 1]: the tokens' log p, 0 where there is none; rounded once, from a sum of fp32
 *                exponentials that is off by less than 2^-22 (30 + classes / 200) of it
 *   accepted_dev [sequences]
 * A logit at or below -1e30 counts as not allowed.  A row without an allowed class, or with NaN or +inf among
 * them, rejects its draft; where it is row n, its token is -1 with log p -inf or NaN.
 * temperature 2^-126 .. 1e27.  workspace_dev: 16-byte aligned, of hier_avg_verify_workspace's bytes.
 * Errors: HA_EINVAL, HA_EUNSUPPORTED for 2^26 rows or 2^24 sequences, HA_ENOMEM, HA_ECUDA. */
int hier_avg_verify_workspace(int64_t sequences, int drafts, int64_t* bytes);
int hier_avg_verify_drafts(const void* logits_dev, int type, int64_t sequences, int drafts, int64_t classes,
                           int64_t logits_seq, int64_t logits_row, const void* drafts_dev, int draft_bytes,
                           const float* uniform_dev, const float* noise_dev, int64_t noise_ld, const void* probs_dev,
                           int probs_type, int64_t probs_seq, int64_t probs_row, const uint8_t* allowed_dev,
                           int64_t allowed_seq, int64_t allowed_row, double temperature, int32_t* tokens_dev,
                           int32_t* accepted_dev, float* logp_dev, void* workspace_dev,
                           int64_t workspace_bytes, void* stream);

/* Synchronise `stream` and report a bounded wait inside a grouped product that ran out on
 * this device (HA_ETIMEOUT, once; the outputs are then invalid) or an asynchronous error.
 * The device has one word for all streams: another stream's wait that has run out by then
 * is reported, and cleared, too. */
int hier_avg_operator_check(void* stream);

const char* hier_avg_strerror(int status);
const char* hier_avg_last_error(const hier_avg* h);

#ifdef __cplusplus
}
#endif

#endif /* HIER_AVG_H */
