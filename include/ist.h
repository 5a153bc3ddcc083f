/*
 * libist — one round of Independent Subnet Training (IST, arXiv 1910.02120) on one GPU.
 *
 * A round (Sec. 2.1 "Methodology" of the paper): the hidden neurons of a fully connected
 * network are randomly partitioned into S disjoint groups ("Constructing Subnets"), every
 * subnet takes the weight slices its neurons select, trains for K iterations of local SGD
 * without talking to the others ("Training Subnets"; K is the paper's J), and the slices are
 * copied back into the full network.  The paper places the S subnets on S machines; here they
 * are S groups of one grouped computation on a single device.
 *
 * Conventions
 *   - C ABI, no exceptions.  Every call returns ist_status (0 = IST_OK, < 0 = error) unless
 *     stated otherwise; ist_last_error() gives a human-readable message for the last failure.
 *   - "dev" pointers are CUDA device pointers, "host" pointers are ordinary host memory.
 *   - The library allocates no device memory.  The caller owns the full network, the inputs,
 *     the outputs and one workspace blob (size from ist_workspace_bytes) that must stay alive
 *     and untouched from ist_create to ist_destroy.
 *   - All device work is enqueued on the stream given to ist_create, in call order, and is
 *     asynchronous to the host.  Only ist_sync_status() synchronises.
 *   - Network layout: layer_dims = {N_0, ..., N_t}; layer l (1..t) has W_l row-major
 *     [N_{l-1}][N_l] fp32 (y = x * W_l + b_l) and b_l [N_l] fp32.  Hidden layers use ReLU;
 *     the loss is the softmax cross-entropy averaged over the minibatch.  (The paper fixes
 *     neither the loss nor biases; these are this library's reading.)
 *   - Call order: ist_create -> ist_bind_weights -> { ist_partition -> ist_local_steps* ->
 *     ist_reassemble }* ; ist_eval any time the network is bound and not partitioned.
 *     Between ist_partition and ist_reassemble the caller must not write the bound weights.
 *   - One process drives one device (kernel attributes and launch limits are looked up once
 *     per process, on the device current at the first call); several contexts on that device
 *     are fine, and calls on one context must not overlap in time.  Calls may come from any
 *     host thread, including one that has made no CUDA call before.
 */
#ifndef IST_H_
#define IST_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ist_ctx ist_ctx; /* opaque, host object */
typedef int32_t ist_status;

enum {
  IST_OK = 0,
  IST_ERR_ARG = -1,            /* null pointer, size out of range, misaligned pointer */
  IST_ERR_STATE = -2,          /* call out of order */
  IST_ERR_WORKSPACE = -3,      /* workspace too small or misaligned */
  IST_ERR_CUDA = -4,           /* a CUDA runtime call failed */
  IST_ERR_DEVICE_CHECK = -5,   /* a device-side bounds check tripped (label / column / index) */
  IST_ERR_DEVICE_TIMEOUT = -6, /* a bounded device-side wait gave up */
  IST_ERR_UNSUPPORTED = -7     /* valid request this build cannot serve */
};

/* Operand precision of the local steps.  Master weights are fp32 in both modes. */
enum { IST_FP32 = 0, IST_BF16 = 1 };

/* Input kinds. */
enum { IST_X_DENSE_F32 = 0, IST_X_DENSE_BF16 = 1, IST_X_CSR = 2 };

/*
 * Minibatches for ist_local_steps / ist_eval.  X is logically [S][K][batch][N_0]: subnet s at
 * local step k reads rows  r0 = s*stride_subnet + k*stride_step ... r0 + batch - 1  (strides in
 * rows; 0 means "the same rows again").  The paper gives every site its own data and draws a
 * minibatch per iteration (Sec. 2.1); the two strides express that.
 *   dense : `dense` points at row-major rows of N_0 elements (fp32 or bf16), device memory.
 *           bf16 rows need N_0 % 8 == 0 and a 16-byte aligned base.
 *   CSR   : row_ptr [rows+1] (absolute offsets into col/val), col [nnz] (0 <= col < N_0,
 *           distinct inside a row), val [nnz] fp32; all device memory.
 * ist_eval ignores the strides and reads rows 0..n-1.
 */
typedef struct ist_input {
  int32_t kind;
  int32_t batch;
  const void* dense;
  const int32_t* row_ptr;
  const int32_t* col;
  const float* val;
  int64_t stride_subnet;
  int64_t stride_step;
} ist_input;

/*
 * Bytes of device workspace a context of this shape needs (0 on invalid arguments).
 * layer_dims: host, n_dims = t+1 entries, each >= 1.  S >= 1 subnets (S = 1 if t = 1),
 * S <= every hidden N_l.  1 <= max_batch <= 65535: largest `batch` later passed in ist_input
 * (ist_eval processes its rows in chunks of max_batch).
 */
size_t ist_workspace_bytes(const int64_t* layer_dims, int n_dims, int S, int precision,
                           int max_batch, int input_is_csr);

/*
 * Sec. 2.1 "Constructing Subnets" says only that each hidden neuron is assigned uniformly at
 * random to one of the n sites; it does not say whether group sizes are fixed.  Two readings:
 * IST_PART_BALANCED (what ist_workspace_bytes / ist_create use): the rule stated at ist_partition,
 * equal group sizes.  IST_PART_IID: every neuron picks its subnet independently (App. A:
 * probability 1/n each): group of neuron i = floor(key_i * S / 2^64) with the same keys, indices
 * ascending inside a group; group sizes are Binomial(N_l, 1/S) and a group may be empty.  The
 * packed layout then has room for ceil(N_l/S) + ceil(7 * sqrt(N_l (1/S)(1 - 1/S))) + 8 neurons
 * per subnet and hidden layer (at most N_l); ist_partition returns IST_ERR_UNSUPPORTED, without
 * enqueueing anything, for a seed whose draw does not fit (probability below 1e-11 per group), and
 * computes the group sizes on the host (N_l hash evaluations per hidden layer and call).
 */
#define IST_PART_BALANCED 0
#define IST_PART_IID 1
size_t ist_workspace_bytes2(const int64_t* layer_dims, int n_dims, int S, int precision,
                            int max_batch, int input_is_csr, int partition_rule);
ist_status ist_create2(ist_ctx** out, const int64_t* layer_dims, int n_dims, int S, int precision,
                       int max_batch, int input_is_csr, int partition_rule, void* workspace_dev,
                       size_t workspace_bytes, void* cuda_stream);

/*
 * Creates a context for a network of the paper's form (Sec. 2: an input layer, t - 1 hidden
 * layers and an output layer with weight matrices between consecutive layers, trained at n = S
 * sites).  Contexts and workspaces themselves have no counterpart in the paper.
 * workspace_dev: device, 256-byte aligned, >= ist_workspace_bytes(...).
 * cuda_stream: a cudaStream_t (NULL = legacy default stream), borrowed.  The workspace is
 * cleared on this stream.  *out is set only on success; free it with ist_destroy.
 */
ist_status ist_create(ist_ctx** out, const int64_t* layer_dims, int n_dims, int S, int precision,
                      int max_batch, int input_is_csr, void* workspace_dev, size_t workspace_bytes,
                      void* cuda_stream);

/*
 * The full network the rounds act on (Sec. 2.1: the model the subnets are cut from and copied
 * back into).  W_dev / b_dev: host arrays of t device pointers
 * (W_l [N_{l-1}][N_l] fp32, b_l [N_l] fp32), borrowed until ist_destroy or the next bind.
 */
ist_status ist_bind_weights(ist_ctx* ctx, float* const* W_dev, float* const* b_dev);

/*
 * Sec. 2.1 "Constructing Subnets" + distribution of the slices.  Draws a fresh partition of
 * every hidden layer from `seed` and gathers each subnet's slices into the workspace:
 * subnet s owns W_1[:, G_1^s], W_l[G_{l-1}^s, G_l^s] for 1 < l < t, W_t[G_{t-1}^s, :], the
 * hidden biases of its neurons and its own copy of the output bias (App. A: each neuron in
 * exactly one subnet; its footnote: a subnet's weight slices leave out everything that belongs
 * to neurons the subnet does not own).
 * Partition rule (the paper states only that the assignment is uniform): neuron i of hidden layer l
 * gets the i-th output of a SplitMix64 generator seeded with the l-th output of a SplitMix64
 * generator seeded with `seed`; neurons are ranked by (key, index); group g takes the next
 * floor(N_l/S) (+1 if g < N_l mod S) ranks; indices are ascending inside a group.
 */
ist_status ist_partition(ist_ctx* ctx, uint64_t seed);

/*
 * Copies the current partition of hidden layer `hidden_layer` (1..t-1) out, i.e. the membership
 * indicators of App. A as index lists (group s = the neurons j with m^(s)_{l,j} = 1):
 * idx_out_dev [N_l] int32 (group-major, ascending inside a group), off_out_dev [S+1] int32.
 */
ist_status ist_get_partition(ist_ctx* ctx, int hidden_layer, int32_t* idx_out_dev,
                             int32_t* off_out_dev);

/*
 * Copies subnet s's current fp32 master slice of layer l (1..t) out, densely:
 * W_out_dev [rows][cols] with rows = |G_{l-1}^s| (N_0 for l = 1), cols = |G_l^s| (N_t for
 * l = t); b_out_dev [cols].  Either pointer may be NULL.  Needs a partition in place.
 */
ist_status ist_get_subnet_params(ist_ctx* ctx, int layer, int s, float* W_out_dev,
                                 float* b_out_dev);

/*
 * Shape of subnet s's slice of layer l (1..t) under the partition in place (Sec. 2.1; Sec. 2.3
 * counts these sizes): *rows_out_host = |G_{l-1}^s| (N_0 for l = 1), *cols_out_host = |G_l^s|
 * (N_t for l = t).  Host outputs, either may be NULL.  These are the extents
 * ist_get_subnet_params writes.  Needs a partition in place (IST_ERR_STATE otherwise).
 */
ist_status ist_subnet_slice_shape(ist_ctx* ctx, int layer, int s, int64_t* rows_out_host,
                                  int64_t* cols_out_host);

/*
 * Sec. 2.1 "Training Subnets": K iterations of local SGD on every subnet, no exchange.
 * Step k of subnet s: forward (App. A Eq. (2) on the slice, without the n^2 factor, as
 * Sec. 2.2 removes it), mean softmax cross-entropy against y, backward, w <- w - lr * grad
 * with all gradients taken at the pre-update weights.
 * y_dev: int32 labels addressed like X rows (row r -> y_dev[r]), 0 <= y < N_t.
 * loss_out_dev: [S*K] fp32, loss_out[s*K + k] = loss of subnet s before the update of step k
 * (may be NULL).  1 <= K.  X->batch <= max_batch.
 */
ist_status ist_local_steps(ist_ctx* ctx, const ist_input* X, const int32_t* y_dev, float lr, int K,
                           float* loss_out_dev);

/*
 * Sec. 2.2, "IST for other architectures": when only the fully connected part of a network is
 * partitioned, the part in front of it (a convolutional trunk, which every site holds whole and
 * trains by local SGD) needs the gradient of each subnet's loss with respect to that subnet's
 * inputs.  Same as ist_local_steps, and in addition
 * dx_out_dev (device, fp32, not NULL): rows addressed exactly like the rows of X (row r of X ->
 * row r of dx_out_dev, N_0 floats each, so the buffer spans as many rows as X does); the row of
 * subnet s, step k, sample b receives d(loss[s][k]) / d(that input row) = delta_1 W_1^T on the
 * subnet's slice, taken at the weights step k starts from.  Rows of X that no step reads are not
 * written.  Dense inputs only (IST_ERR_UNSUPPORTED for CSR); on the bf16 path N_0 must be a
 * multiple of 4.  With K > 1 the later steps' gradients belong to inputs the trunk produced
 * before its own update: the usual call has K = 1.
 */
ist_status ist_local_steps_dx(ist_ctx* ctx, const ist_input* X, const int32_t* y_dev, float lr, int K,
                              float* loss_out_dev, float* dx_out_dev);

/*
 * Training the S subnets at several sites (Sec. 2.1 "Distributing Subnets": every subnet goes to
 * its own compute node; Sec. 2.3: only the slices travel).  A context may own only subnets
 * first .. first + count - 1: ist_partition then draws the whole partition (it is cheap and every
 * site needs the same one) but gathers only the owned subnets' slices, and ist_local_steps trains
 * only those; the other subnets are trained by other contexts (other GPUs, one process each) that
 * hold a copy of the same full network and draw the same partition (same seed).  Before
 * ist_reassemble every context must hold all S trained slices: ist_packed_layer gives the device
 * address of layer l's packed fp32 slices ([S][*master_bytes_per_subnet], subnet s at byte
 * offset s * bytes) and of its packed biases, so that the caller can exchange them (one
 * all-gather per layer over the subnet dimension, each site contributing its own `count` slabs).
 * ist_reassemble writes all S slabs back, whoever trained them.
 * On the bf16 path the slices are otherwise kept as bf16 operands and the masters' low halves, which a
 * weight update moves with 8 bytes per weight instead of 10; the first ist_packed_layer call makes them
 * fp32 in place (enqueued on the context's stream) and the context keeps fp32 slices from then on.  The values
 * are the same either way, bit for bit; only a NaN may come back as another NaN from the operand form.
 * In ist_local_steps the inputs and losses are then addressed by the local subnet index
 * (0 .. count-1): rows start at i * stride_subnet, loss_out_dev holds count * K values.
 * Default range: all S subnets.  Not allowed while a partition is in place.
 */
ist_status ist_set_subnet_range(ist_ctx* ctx, int first, int count);
ist_status ist_packed_layer(ist_ctx* ctx, int layer, void** master_dev, size_t* master_bytes_per_subnet,
                            void** bias_dev, size_t* bias_bytes_per_subnet);

/*
 * Sec. 2.1 "Training Subnets", last step: the trained slices go back into the full network; the
 * groups are disjoint, so no two subnets write the same entry.
 * Writes every trained slice to the positions it was gathered from; entries of middle layers
 * whose row group differs from their column group are not written.  The output bias, the one
 * parameter all subnets hold, becomes b + (sum_s (b^(s) - b)) / S (its mean over the copies).
 * Afterwards the context is back in the "bound" state.
 */
ist_status ist_reassemble(ist_ctx* ctx);

/*
 * Full-width forward pass of the bound network (the deployed model, Sec. 2.2) over n rows:
 * mean softmax cross-entropy -> *mean_loss_out_dev (fp32), number of rows whose arg-max
 * (lowest index on ties) equals the label -> *n_correct_out_dev (int64).  Computed in fp32.
 */
ist_status ist_eval(ist_ctx* ctx, const ist_input* X, const int32_t* y_dev, int64_t n,
                    float* mean_loss_out_dev, int64_t* n_correct_out_dev);

/*
 * Sec. 2.2 "Correcting Distributional Shift", second remedy: every hidden neuron's input is
 * standardised over the minibatch before the non-linearity,
 *   zh = (z - mean_b z) / sqrt(var_b z + eps),  a = max(zh, 0),
 * per subnet and neuron, with the biased (1/batch) variance and no learned scale or shift (the
 * paper fixes neither eps nor the variance estimator), and the backward pass differentiates
 * through it:  d_z = (d_zh - mean_b d_zh - zh * mean_b(d_zh * zh)) / sigma.
 *
 * ist_norm_workspace_bytes: bytes of a second device blob that holds the fp32 pre-activations
 * of the hidden layers ([S][max_batch][n_l] per layer) and the statistics.
 * ist_enable_normalization: switches the context to this mode for all later calls (there is no
 * way back).  norm_workspace_dev: device, 256-byte aligned, at least that many bytes, borrowed
 * until ist_destroy; it is cleared on the context's stream.  eps > 0.  Not allowed while a
 * partition is in place.
 * ist_calibrate: the deployment statistics of Sec. 2.2: mean and standard deviation of every
 * hidden neuron's input over rows 0..n-1 of X (1 <= n <= max_batch, fp32 or CSR rows), computed
 * with the bound full network layer by layer in fp32.  ist_eval then standardises with these
 * stored values.  ist_reassemble and ist_bind_weights discard the statistics (they belong to the
 * weights they were taken with); in this mode ist_eval without valid statistics returns
 * IST_ERR_STATE.
 */
size_t ist_norm_workspace_bytes(const ist_ctx* ctx);
ist_status ist_enable_normalization(ist_ctx* ctx, float eps, void* norm_workspace_dev,
                                    size_t norm_workspace_bytes);
ist_status ist_calibrate(ist_ctx* ctx, const ist_input* X, int64_t n);

/* Waits for the stream and returns the sticky device status (IST_OK, IST_ERR_DEVICE_CHECK,
 * IST_ERR_DEVICE_TIMEOUT or IST_ERR_CUDA). */
ist_status ist_sync_status(ist_ctx* ctx);

/*
 * Self-test of the device-side error path (no counterpart in the paper).  Every wait inside the
 * tensor-core kernels is bounded: after its limit it records IST_ERR_DEVICE_TIMEOUT in the status
 * word and the kernel returns.  This call enqueues, on the context's stream, a one-block kernel that
 * waits with the same routine on a barrier nothing ever signals, for limit_cycles SM clock cycles
 * (1 .. 2e9, i.e. at most about a second), so that the wait must give up.  Afterwards
 * ist_sync_status returns IST_ERR_DEVICE_TIMEOUT for this context (the status word is sticky: create
 * a new context to go on); the stream and the device stay usable.  Returns IST_ERR_ARG for a limit
 * outside the range, IST_ERR_CUDA if the launch fails.
 */
ist_status ist_selftest_wait_expiry(ist_ctx* ctx, int64_t limit_cycles);

/*
 * Measurement aid (no counterpart in the paper).  Kernel classes of a round, in the order a
 * round runs them.  With profiling enabled every group of launches of one class is bracketed
 * by a pair of CUDA events on the context's stream; ist_profile_read synchronises and returns
 * the number of kernels launched and the summed device time of that class since profiling was
 * enabled.  Enabling clears earlier records.  The events cost a few microseconds each, so
 * throughput should be timed with profiling off.
 */
enum {
  IST_K_PARTITION = 0, /* keys, ranks, index lists */
  IST_K_GATHER = 1,    /* full network -> packed slices (+ bf16 copies) */
  IST_K_STAGE = 2,     /* fp32 input rows -> bf16 staging */
  IST_K_FWD = 3,       /* forward GEMMs with bias / ReLU / logits epilogues */
  IST_K_LOSS = 4,      /* softmax cross-entropy, loss reduction */
  IST_K_DX = 5,        /* delta_{l-1} GEMMs with the ReLU mask epilogue */
  IST_K_DW_SGD = 6,    /* weight-gradient GEMMs with the fused SGD update */
  IST_K_BIAS_SGD = 7,  /* bias gradient and update */
  IST_K_SPMM = 8,      /* sparse first layer: forward, backward + update */
  IST_K_SCATTER = 9,   /* packed slices -> full network */
  IST_K_EVAL = 10,     /* full-width evaluation */
  IST_K_NORM = 11,     /* batch standardisation, forward and backward (Sec. 2.2) */
  IST_K_COUNT = 12
};
ist_status ist_profile(ist_ctx* ctx, int enable);
ist_status ist_profile_read(ist_ctx* ctx, int kernel_class, int64_t* launches_out_host,
                            double* ms_out_host);

/*
 * Partition of one hidden layer without a context, a workspace or any allocation.  (The paper
 * has no counterpart; this is a service entry point of the library.)
 *
 * For callers that cannot obtain device memory at the time they need a partition: code running
 * inside a host application that gave out its device-memory budget at start-up and forbids
 * allocation afterwards, or a process that only wants the index lists (for example to decide
 * which weight slices to fetch) and has no room for an ist_ctx workspace.  The caller passes
 * only its own outputs; the kernels' intermediate arrays live in a device array that is part of
 * the library image, 2 MB that every GPU loading the library holds until exit.
 *
 * Result: exactly the partition ist_partition(seed) draws for hidden layer `hidden_layer`
 * (1-based) when that layer has n_neurons neurons and the network is split into S subnets:
 * idx_out_dev [n_neurons] int32 (group-major, ascending inside a group), off_out_dev [S+1].
 * Work is enqueued on cuda_stream (a cudaStream_t, NULL = default stream), asynchronously.
 *
 * Limits: n_neurons <= IST_STATIC_MAX_NEURONS and S <= IST_STATIC_MAX_SUBNETS, otherwise
 * IST_ERR_UNSUPPORTED and nothing is enqueued.  IST_ERR_ARG for null outputs, S < 1,
 * S > n_neurons or hidden_layer outside 1..62.  The call performs no cudaMalloc / cudaFree and
 * calls no allocating routine.
 *
 * The first call on a device looks up the device address of the built-in array (a host-side
 * set-up step): make that first call before starting any stream capture.
 * All calls on a device share the one array, which keeps the previous call's contents; the
 * entry point clears what has to start at zero.  Two calls whose kernels can overlap on the
 * GPU (different streams without an ordering between them) race on it: order them.
 */
#define IST_STATIC_MAX_NEURONS 65536
#define IST_STATIC_MAX_SUBNETS 64
ist_status ist_partition_layer_static(uint64_t seed, int hidden_layer, int64_t n_neurons, int S,
                                      int32_t* idx_out_dev, int32_t* off_out_dev, void* cuda_stream);

/*
 * Device-side status of ist_partition_layer_static on the current device (no counterpart in the
 * paper).  Its kernels check every index they emit against [0, n_neurons) and record a failure
 * in a status word at the start of the built-in array; each call of the entry point clears the
 * word first, so this reports on the most recent call.  Waits for cuda_stream (the stream that
 * call used), copies the word to the host and returns IST_OK or IST_ERR_DEVICE_CHECK
 * (IST_ERR_CUDA if the copy fails).  Allocates nothing.  Before the first
 * ist_partition_layer_static call on the device it returns IST_OK.
 */
ist_status ist_static_partition_status(void* cuda_stream);

/* Number of kernels this context has launched so far (host counter). */
int64_t ist_kernel_launches(const ist_ctx* ctx);

/* Message for the most recent failing call on this context ("" if none).  ctx may be NULL,
 * in which case the message of the last failing ist_create, or of the last failing call of those
 * below that take no context, on this thread is returned. */
const char* ist_last_error(const ist_ctx* ctx);

/*
 * Operators for the part of a network that stands in front of the partitioned layers (Sec. 2.2,
 * "IST for other architectures": a trunk that every site holds whole).  The paper has no counterpart;
 * ist_local_steps_dx gives such a trunk its gradient, these calls normalise what it hands to the head
 * and update its parameters.  They take no context.  Work is enqueued on cuda_stream (a cudaStream_t,
 * NULL = legacy default stream) of the current device, which may be another one from call to call (launches are sized
 * for GPUs of one kind), asynchronously, and may be captured into a
 * graph; nothing is allocated and nothing is kept from one call for the next.  Two calls, and two graphs, that may
 * run at the same time need workspaces of their own.  Invalid arguments return an error and enqueue
 * nothing; ist_last_error(NULL) has the message.
 */

/* Element types. */
enum { IST_T_F32 = 0, IST_T_BF16 = 1 };

/*
 * Layer normalisation of rows.  x_dev: `rows` rows of `cols` elements, x_stride elements from one row to the
 * next (>= cols); so are y, dy and dx with theirs.  The rows belong in order to `groups` sites, rows / groups
 * each (rows must be a multiple of groups), and every site has its own weight and bias
 * (weight_dev, bias_dev: [groups][cols] fp32; NULL stands for ones and for zeros).  Per row
 *   mean = sum_j x_j / cols,   rstd = 1 / sqrt(sum_j (x_j - mean)^2 / cols + eps),
 *   y_j = (x_j - mean) * rstd * weight_j + bias_j.
 * mean_out_dev, rstd_out_dev: [rows] fp32 for the backward pass, either may be NULL.  Statistics are taken
 * in fp32 or wider from the elements' values; y is rounded once, to nearest even.  A row that holds an infinity or
 * a NaN comes out as NaN, other rows are not touched by it.  Sums over a row of up to 65,536 columns are fp32 sums and have to
 * stay within that type's range: the values', and that of the squares of their differences from the mean as it is
 * rounded.  Magnitudes up to 1e16 are always fine; rows of larger values may come out as NaN or as the bias.
 * rows = 0 is allowed.  0 < eps < inf.
 * 1 <= cols <= 2^30, 0 <= rows <= 2^31 - 65536, 1 <= groups < 2^31.  Outputs must not overlap inputs or one another
 * (rows of one buffer that interleave without sharing elements are fine if their strides are the same number of bytes; others
 * are refused).  Elements between the rows are left as they are.
 * Very wide rows are shared by several blocks, whose waits for one another are bounded (about a second): a wait that gave up
 * leaves NaN in its row and in those that its block takes after it, and ist_layer_norm_status tells of it.
 */
ist_status ist_layer_norm_forward(const void* x_dev, int x_type, int64_t x_stride, int64_t rows, int64_t cols,
                                  int groups, const float* weight_dev, const float* bias_dev, float eps, void* y_dev,
                                  int y_type, int64_t y_stride, float* mean_out_dev, float* rstd_out_dev,
                                  void* cuda_stream);

/*
 * The way back, from what the forward pass read and returned: with h = (x - mean) * rstd and g = dy * weight,
 *   dx_j = rstd * (g_j - sum_i g_i / cols - h_j * sum_i g_i h_i / cols)   (x's type),
 *   dweight = sum over the site's rows of dy * h,   dbias = sum over the site's rows of dy   ([groups][cols] fp32).
 * dx_out_dev, dweight_out_dev and dbias_out_dev may be NULL where they are not wanted (not all three).  The sums over rows
 * are added in an order that depends on shape, types, alignment and the number of the GPU's multiprocessors alone, so results are
 * the same from call to call.  Like those over a row they are fp32 sums and have to stay within that type's range.  rows = 0 gives
 * zeros for dweight and dbias.  workspace_dev: at least ist_layer_norm_workspace_bytes(rows, cols, groups) bytes
 * (0 where none is needed, and on invalid arguments, which the call then refuses), 16-byte aligned; may be NULL where none is needed or neither
 * dweight nor dbias is wanted; its content means nothing before and after the call.
 */
size_t ist_layer_norm_workspace_bytes(int64_t rows, int64_t cols, int groups);
ist_status ist_layer_norm_backward(const void* dy_dev, int dy_type, int64_t dy_stride, const void* x_dev, int x_type,
                                   int64_t x_stride, int64_t rows, int64_t cols, int groups, const float* weight_dev,
                                   const float* mean_dev, const float* rstd_dev, void* dx_out_dev, int64_t dx_stride,
                                   float* dweight_out_dev, float* dbias_out_dev, void* workspace_dev,
                                   size_t workspace_bytes, void* cuda_stream);

/*
 * Waits for cuda_stream and returns IST_ERR_DEVICE_TIMEOUT if a wait of either pass on the current device gave up since
 * this was last asked, else IST_OK (IST_ERR_CUDA if the flag cannot be read).  Not for streams under capture.
 */
ist_status ist_layer_norm_status(void* cuda_stream);

/*
 * Self-test of that path (no counterpart in the paper): layer norm of rows x [rows][cols] without weights, fp32, where blocks
 * withhold their sums from one another, so that the waits for limit_cycles SM clock cycles (1 .. 2e9) must give up.  dy_dev
 * NULL: the forward pass, out = y.  Else the way back, out = dx, with stats_dev = [rows] means and [rows] reciprocal deviations.
 * 16385 <= cols <= 65536 (rows that blocks share), 1 <= rows <= 65536.  All of out becomes NaN and ist_layer_norm_status
 * returns IST_ERR_DEVICE_TIMEOUT; stream and device stay usable.
 */
ist_status ist_selftest_layer_norm_wait(const float* x_dev, const float* dy_dev, const float* stats_dev, int64_t rows,
                                        int64_t cols, float* out_dev, int64_t limit_cycles, void* cuda_stream);

/*
 * One AdamW step over many tensors.  For every parameter, with gradient g, step number t (1 for the first) and
 * clipping factor c:
 *   g' = c g,   m = beta1 m + (1 - beta1) g',   v = beta2 v + (1 - beta2) g'^2,
 *   p = p - lr weight_decay p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps),
 * and, where param_bf16 is given, param_bf16 = p rounded to bf16 (to nearest even).
 * c = max_norm / norm if max_norm > 0 and norm > max_norm, else 1; norm is the square root of the sum of g^2 over all
 * tensors of the call.  A norm that is not finite is no error: the factor follows from the same rule (0 for an infinite norm,
 * 1 for a NaN), and what is not finite in the gradients reaches the parameters and states that it belongs to.
 *
 * States (state_bits): 32: exp_avg, exp_avg_sq are fp32 [n] (m and v).  8: they are one byte per value,
 * and the blocks of IST_ADAMW_BLOCK consecutive values of a tensor share one int16 each in exp_avg_base and
 * exp_avg_sq_base ([ceil(n / IST_ADAMW_BLOCK)]): a code c > 0 of 8 bits (v), or of the lower 7 bits (m, whose bit 7 is the
 * sign), is the fp32 number with the bit pattern (base + c) << 20, code 0 is zero, and the largest code (255, 127) stands for a value
 * that is not finite (infinity for v, NaN for m).  So values have 3 bits behind the leading one, and a block reaches 2^31 (v)
 * or 2^15 (m) below its largest value, from which the base is taken anew in every step.  Zeros everywhere are the states
 * before the first step.  The parameter is updated from m and v before they are rounded.  Rounding is random and keeps the mean (to
 * nearest, an average that moves by a thousandth per step would stand still): a value's fp32 bit pattern plus 20 random
 * bits is cut at bit 20; the random bits are 16 r + 8, with r for elements 2 i and 2 i + 1 of tensor j from word w = the (i+1)-th output
 * of a SplitMix64 generator seeded with the (j+1)-th output of one seeded with the t-th output of one seeded with `seed`:
 * bits 0..15 (m) and 16..31 (v) of w for element 2 i, 32..47 and 48..63 for element 2 i + 1.  What falls below the block's
 * range becomes zero (m) or the smallest code (v: a divisor must not vanish).
 *
 * A tensor with n = 0 or grad = NULL is passed over (its number j still counts).  The tensors' arrays must not overlap one
 * another; gradients, which are only read, may overlap one another, and one may be the very array of its own parameter.  Arrays need the alignment of their elements; arrays that start on 16 bytes (on 4
 * bytes those of 1-byte codes) are faster.  The table of tensors and the arguments are read during the call.
 * step, lr: of this step.  A graph replays the arguments of its capture, so for a captured step they may come from
 * the device instead: step_dev (int64), lr_dev (fp32), not NULL, are read when the kernels run, in place of step and lr.
 * norm_out_dev (may be NULL): receives the norm (fp32) if max_norm > 0.
 * workspace_dev: with max_norm > 0 at least ist_adamw_workspace_bytes(count) bytes, 16-byte aligned; else not
 * needed.  Its content means nothing before and after the call.
 * Needs 0 <= beta < 1 for both, 2^-126 <= eps <= 2^125, step >= 1, finite lr and weight decays, max_norm >= 0 (infinity: no clipping, but the norm is taken), at most 2^40 values.
 */
#define IST_ADAMW_BLOCK 128
typedef struct ist_adamw_tensor {
  float* param;
  const void* grad;
  void* exp_avg;
  void* exp_avg_sq;
  int16_t* exp_avg_base;    /* 8 bits only */
  int16_t* exp_avg_sq_base; /* 8 bits only */
  void* param_bf16;         /* may be NULL */
  int64_t n;
  double weight_decay;
} ist_adamw_tensor;
typedef struct ist_adamw_args {
  double lr, beta1, beta2, eps;
  double max_norm; /* 0: no clipping */
  int64_t step;
  uint64_t seed; /* 8 bits only */
  int32_t state_bits;
  int32_t grad_type;
  const int64_t* step_dev; /* may be NULL */
  const float* lr_dev;     /* may be NULL */
  float* norm_out_dev;     /* may be NULL */
} ist_adamw_args;
size_t ist_adamw_workspace_bytes(int64_t count);
ist_status ist_adamw_step(const ist_adamw_tensor* tensors_host, int64_t count, const ist_adamw_args* args,
                          void* workspace_dev, size_t workspace_bytes, void* cuda_stream);

/*
 * The values that 8-bit states stand for (to look at, or to keep elsewhere): n codes and ceil(n / IST_ADAMW_BLOCK) bases
 * each of first and second moments, as above, become n fp32 or bf16 values (out_type; exact in both).  Either pair of
 * outputs and its inputs may be NULL.
 */
ist_status ist_adamw_state_values(const uint8_t* exp_avg, const int16_t* exp_avg_base, const uint8_t* exp_avg_sq,
                                  const int16_t* exp_avg_sq_base, int64_t n, int out_type, void* exp_avg_out_dev,
                                  void* exp_avg_sq_out_dev, void* cuda_stream);

/* Frees the host object.  Does not touch device memory; pending work keeps running. */
void ist_destroy(ist_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* IST_H_ */
