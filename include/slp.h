/*
 * slp -- segment-wise training with synthetic intermediate labels on one AMD
 * MI355X (gfx950).  C ABI of the hot path of "Partitioned Neural Network
 * Training via Synthetic Intermediate Labels" (arXiv 2403.11204): the independent
 * training step of one network segment.
 *
 * Conventions
 *   - every function returns SLP_OK (0) or a negative slp_status; nothing throws
 *     across this boundary; slp_last_error() gives a thread-local message;
 *   - "device" pointers are HIP device addresses on the current device, "host"
 *     pointers are ordinary host memory; the library allocates NO device memory:
 *     every device byte it uses is handed in by the caller (slp_segment_bind);
 *   - slp_stream is a hipStream_t passed as void* (NULL = the default stream);
 *     calls that take a stream are asynchronous on it unless stated otherwise;
 *   - matrices are row-major; a weight matrix is [out][in] as in the paper's
 *     parameter count (in+1)*out (Sec. 3);
 *   - a label table is stored [classes][dim]: row j is the synthetic intermediate
 *     label of class j (the paper's SIL is the transpose, one column per class).
 *   - argument validation happens on the host before any device work is queued: a call
 *     that returns an error has launched nothing;
 *   - calls on ONE handle must not overlap in time (they share its workspace); different
 *     handles are independent and may run concurrently on different streams (Sec. 2.1:
 *     partitions are independent jobs).  A training step may also use a second stream that
 *     the handle owns (default priority) for parameter updates; it is forked from and
 *     joined back into `stream` inside the call, so `stream` alone orders everything.
 */
#ifndef SLP_H
#define SLP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct slp_segment slp_segment;
typedef void* slp_stream;

typedef enum {
  SLP_OK = 0,
  SLP_ERR_ARG = -1,    /* null pointer, unknown enum value, non-positive size */
  SLP_ERR_SHAPE = -2,  /* sizes that do not fit each other or the handle's limits */
  SLP_ERR_ALLOC = -3,  /* a caller-provided buffer is too small or misaligned */
  SLP_ERR_DEVICE = -4, /* the HIP runtime reported an error */
  SLP_ERR_STATE = -5   /* call made before the state it needs exists */
} slp_status;

/* label distributions: Eq. 1 of the paper is SLP_UNIFORM01 (kappa * U[0,1)) */
typedef enum { SLP_UNIFORM01 = 0, SLP_UNIFORM_PM1 = 1, SLP_NORMAL = 2, SLP_BINARY_PM1 = 3 } slp_dist;
typedef enum { SLP_F32 = 0, SLP_BF16 = 1 } slp_dtype;
/* Sec. 3: ReLU after every layer except the network's last one.  A non-final
 * segment ends at a cut and keeps its ReLU (SLP_RELU_ALL); the final segment
 * ends in the identity (SLP_RELU_HIDDEN_IDENTITY_LAST). */
typedef enum { SLP_RELU_ALL = 0, SLP_RELU_HIDDEN_IDENTITY_LAST = 1 } slp_act;
/* Sec. 2: a non-final segment regresses on the synthetic label of the sample's
 * class (mean squared error over batch x width); the final segment is trained on
 * the true classes (softmax cross-entropy, mean over the batch). */
typedef enum { SLP_MSE_SIL = 0, SLP_SOFTMAX_XENT = 1 } slp_loss;

typedef struct {
  int dtype;      /* slp_dtype: SLP_F32 = everything float32; SLP_BF16 = bf16 weights copy,
                     activations and dZ with float32 accumulation, float32 master weights,
                     gradients, momentum and biases */
  int max_batch;  /* largest batch a step or forward call may pass */
  float lr;       /* SGD learning rate (Sec. 3 uses 0.01) */
  float momentum; /* SGD momentum (Sec. 3 uses 0.9); 0 = plain SGD */
  int input_grad; /* 1: the segment can also return d loss / d input (slp_segment_input_grad); costs a
                     transposed copy of the first layer's weights and one input-sized buffer */
} slp_opts;

const char* slp_last_error(void);

/* ---- synthetic intermediate labels (Sec. 2, Eq. 1) --------------------------------
 * Writes T[classes][dim] (dense, row-major, dtype dt) to the caller-owned device
 * buffer `table`.  Entry (j,i) is a pure function of (seed, j, i, dist, kappa):
 * Philox4x32-10 with key = seed and counter (i, j, 0, 0), then a fixed float32
 * transform; kappa only scales SLP_UNIFORM01.  Bit-exact against the CPU
 * definition.  A bf16 table is the float32 value rounded to nearest even. */
int slp_make_synthetic_labels(uint64_t seed, int classes, int dim, int dist, float kappa,
                              void* table /*device*/, int dt, slp_stream stream);

/* ---- inputs of an interior segment in the simultaneous variant (Sec. 2, the
 * variant that trains every partition at once, where an interior partition takes
 * synthetic labels as its inputs as well as its targets) ----------------------------
 * out[n][i] = table[y[n]][i] + sigma * N(0,1), noise counter = global sample index
 * first_sample + n (Philox stream 2).  table: float32 [classes][dim] device;
 * y: int32 [batch] device, each in [0,classes) (clamped into range on the device);
 * out: [batch][dim] of dtype dt, device, caller-owned. */
int slp_make_segment_inputs(uint64_t seed, const float* table /*device*/, int classes, const int32_t* y /*device*/,
                            int64_t first_sample, int batch, int dim, float sigma,
                            void* out /*device*/, int dt, slp_stream stream);

/* ---- segment handle (Sec. 2: one partition; Sec. 2.1: its own hyper-parameters) ----
 * widths[0..n_widths-1] = input width then the width of every layer, n_widths >= 2.
 * The handle is host memory owned by the library until slp_segment_destroy.
 * Errors: SLP_ERR_ARG (null pointers, n_widths < 2 or > 65, a width outside [1, 2^20], unknown enum, max_batch
 * outside [1, 2^24], lr < 0, momentum outside [0,1)); SLP_ERR_SHAPE when a matrix cannot be
 * addressed with 32-bit byte offsets: a weight matrix (float32) or an activation matrix (max_batch x width
 * in the handle's dtype, and its transposed copy) of 2 GiB or more, counted with the library's leading
 * dimensions: the row length rounded up to a multiple of 64 elements, plus 192 elements where that row would
 * be a multiple of 4 KB in the handle's dtype. */
int slp_segment_create(const int* widths /*host*/, int n_widths, int act, int loss, const slp_opts* opts /*host*/,
                       slp_segment** out);
void slp_segment_destroy(slp_segment* seg);

/* Bytes of device memory the segment needs: parameters + optimiser state +
 * gradients ("params"), and activations / per-step temporaries ("workspace"). */
size_t slp_segment_param_bytes(const slp_segment* seg);
size_t slp_segment_workspace_bytes(const slp_segment* seg);

/* Hands the two caller-owned device buffers (256-byte aligned, at least the sizes
 * above) to the segment and zero-fills them on `stream`.  They must outlive every
 * later call on the handle; the library never frees them.  Parameters are undefined
 * (zero) until slp_segment_init or slp_segment_set_params on every layer.
 * Errors: SLP_ERR_ARG (null), SLP_ERR_ALLOC (misaligned or too small), SLP_ERR_DEVICE. */
int slp_segment_bind(slp_segment* seg, void* params /*device*/, size_t params_bytes, void* workspace /*device*/,
                     size_t workspace_bytes, slp_stream stream);

/* Initial parameters U(-1/sqrt(fan_in), 1/sqrt(fan_in)) for weights and biases (the
 * default of the framework named in Sec. 2), drawn from Philox stream 1 with
 * counter (in, out, 1, layer), bias at in = fan_in; momentum is reset to zero. */
int slp_segment_init(slp_segment* seg, uint64_t seed, slp_stream stream);

/* Parameter / gradient / momentum exchange, always as dense float32 W[out][in] and
 * b[out] whatever the internal layout; layer in [0, n_widths-2]; on_device selects
 * host or device pointers for W and b; either pointer may be NULL to skip it.  The
 * calls synchronise `stream` before returning when a host pointer is involved.
 * set_params also rebuilds the derived weight copies and leaves momentum alone.
 * Errors: SLP_ERR_ARG (layer out of range), SLP_ERR_STATE (not bound; get_* before any
 * parameters exist), SLP_ERR_DEVICE. */
int slp_segment_set_params(slp_segment* seg, int layer, const float* W, const float* b, int on_device, slp_stream stream);
int slp_segment_get_params(slp_segment* seg, int layer, float* W, float* b, int on_device, slp_stream stream);
int slp_segment_get_grads(slp_segment* seg, int layer, float* dW, float* db, int on_device, slp_stream stream);
int slp_segment_get_momentum(slp_segment* seg, int layer, float* vW, float* vb, int on_device, slp_stream stream);
/* Copies the stored activation A_layer (layer 0 = the ingested input, layer L =
 * the segment's output) of the last step, rows [0,batch), to out[batch][width],
 * dense, in the handle's dtype (device pointer). kind 0 = activation, 1 = dZ (layers 1..L). */
int slp_segment_get_activation(slp_segment* seg, int layer, int kind, int batch, void* out /*device*/, slp_stream stream);

int slp_segment_set_lr(slp_segment* seg, float lr, float momentum);

/* Label table for a SLP_MSE_SIL segment (Sec. 2, first training phase: the left partition is trained against the
 * synthetic intermediate label of each sample's class): float32 [classes][dim] on the device with
 * dim == the segment's last width; caller-owned, must outlive the steps.
 * Errors: SLP_ERR_STATE (the segment's loss is not SLP_MSE_SIL), SLP_ERR_ARG (null table,
 * classes <= 0), SLP_ERR_SHAPE (dim != last width). */
int slp_segment_set_labels(slp_segment* seg, const float* table /*device*/, int classes, int dim);

/* ---- the training step (Sec. 2: first and second training phase; Sec. 3:
 * optimiser and activations) -------------------------------------------------------
 * One pass of forward, loss, backward confined to the segment, and the SGD update
 * for the batch X[batch][widths[0]] (dense, handle dtype, device) with class ids
 * targets[batch] (int32, device).  For SLP_MSE_SIL the ids select rows of the bound
 * label table; for SLP_SOFTMAX_XENT they are the classes (< last width).  Ids are
 * clamped into range on the device and counted (slp_segment_target_errors).  If loss_out is not NULL the mean loss of the
 * batch (before the update) is written there (float32, device).  No host
 * synchronisation; X and targets are only read.  batch may be any value in
 * [1, max_batch]; the means run over the batch actually passed.
 * Errors: SLP_ERR_ARG (null X or targets), SLP_ERR_SHAPE (batch outside [1, max_batch]),
 * SLP_ERR_STATE (not bound, no parameters, SLP_MSE_SIL without a label table),
 * SLP_ERR_DEVICE (a launch failed). */
int slp_segment_step(slp_segment* seg, const void* X /*device*/, const int32_t* targets /*device*/, int batch,
                     float* loss_out /*device, may be NULL*/, slp_stream stream);

/* Class ids are the caller's data: an id outside its range (rows of the label table for SLP_MSE_SIL, the last width
 * for SLP_SOFTMAX_XENT) is clamped into range on the device so that nothing is read out of bounds, and the row is
 * COUNTED: *count_out (host) receives the number of such rows seen by the handle's loss kernels since slp_segment_bind.
 * A non-zero count means steps trained on wrong targets.  Synchronises `stream`.  Errors: SLP_ERR_ARG (null),
 * SLP_ERR_STATE (not bound), SLP_ERR_DEVICE. */
int slp_segment_target_errors(slp_segment* seg, int64_t* count_out /*host*/, slp_stream stream);

/* Forward only (Sec. 2: the stored response of the left partition; joining the
 * partitions): out[batch][last width], dense, handle dtype, device.  Parameters
 * are not changed; the activation workspace is overwritten (X and out themselves are
 * used in place of its first and last entries when their rows are aligned: X with a
 * width that is a multiple of 64 on a 128-byte boundary, out with a width that is a
 * multiple of 8 on a 16-byte boundary).  out may overlap X.  Errors as for the step. */
int slp_segment_forward(slp_segment* seg, const void* X /*device*/, int batch, void* out /*device*/, slp_stream stream);

/* ---- recovery phase (Sec. 5: the left partition is trained some more while the
 * right partition's weights are frozen) ------------------------------------------------
 * slp_segment_input_grad runs forward, the segment's own loss against `targets` and
 * the data gradients of EVERY layer, and writes d loss / d X to dX[batch][widths[0]]
 * (dense, handle dtype, device).  No parameter, momentum or gradient buffer changes:
 * this is the frozen partition.  Needs opts.input_grad = 1 (else SLP_ERR_STATE).
 * slp_segment_step_external is a training step whose output gradient comes from
 * outside: dA_out[batch][last width] (dense, handle dtype, device) = d loss / d (segment
 * output).  dZ_L = dA_out where the last layer's ReLU is active (or everywhere on an
 * identity-last segment), then the usual backward pass and SGD update.  Chaining
 * left.forward -> right.input_grad -> left.step_external is one recovery step. */
int slp_segment_input_grad(slp_segment* seg, const void* X /*device*/, const int32_t* targets /*device*/, int batch,
                           void* dX /*device*/, float* loss_out /*device, may be NULL*/, slp_stream stream);
int slp_segment_step_external(slp_segment* seg, const void* X /*device*/, const void* dA_out /*device*/, int batch,
                              slp_stream stream);

/* ---- launch-bound segments ----------------------------------------------------------
 * A step of a small segment (the paper's own network is 784-80-60 | 60-60-60-47, Sec. 3) is a
 * few dozen kernels of a few microseconds each: the host's launch rate, not the GPU, bounds
 * it.  With graphs on, slp_segment_step captures its launch sequence into a HIP graph the
 * first time it sees a combination (X, targets, batch, loss_out) -- the only arguments the
 * sequence depends on -- and replays that graph, one launch, on every later call with the
 * same combination (up to 16 are kept, least recently used evicted).  Results are those of
 * the eager launches, bit for bit: the same kernels with the same arguments in the same order.
 * Steps of small layers that come to at most 8 launches are launched one by one all the same: that measured faster than
 * starting a graph (784-128-64, batch 64: 4 launches, 18.5 us a step against 25.8).
 * Eager launches are used regardless while launches are being timed (profile hooks on), on the
 * null stream, for the first step of a handle, and when `stream` is already being captured by
 * the caller (the launches then become part of the caller's graph).  slp_segment_set_lr,
 * slp_segment_set_labels and slp_segment_bind drop the captured graphs (after a device
 * synchronisation), because those hold their values.  A caller that keeps passing new
 * combinations would pay a capture per step: after 32 misses in a row the handle returns to
 * eager launches until this function is called again (copy each batch into one fixed buffer
 * and step on that to have a single combination).  Off by default. */
int slp_segment_set_graph(slp_segment* seg, int on);
/* What became of it: *captured = graphs the handle holds now, *replayed = steps it has taken by starting one, the step that
 * captured it included (either pointer, host, may be NULL).  Errors: SLP_ERR_ARG (null handle). */
int slp_segment_graph_stats(const slp_segment* seg, int* captured /*host*/, int64_t* replayed /*host*/);

/* ---- optimiser step inside the weight-gradient product (Sec. 3: SGD with momentum) ----------------------
 * With the fused update on, the matrix product that forms dW_l applies v = mu v + dW; w = w - lr v to the tile of the
 * weight matrix it holds and rewrites the bf16 and transposed copies from there: the gradient is never written to
 * memory and never read back (20 instead of 28 bytes per parameter and step in bf16 mode), and a step of a mid-size
 * segment ends with its last product instead of a tail of update launches.  It pays while the batch is short, whatever the
 * width: at long ones (bf16: from 2300 to 4000 rows on, by the shape) the separate update, which streams beside the next products,
 * is faster.  on = 0: off (default); 1: every layer; 2: the layers with at most 4,194,304 weights; on > 2: the layers with at
 * most `on` weights.  What the switch decides is which gradients are stored.
 * Off or on, layers with fewer than 224 tiles of 128x128 weights take the update inside the product in any case, and so do
 * larger ones at batches up to 2048 (float32 4096; with overlap on below 1400, float32 640) where that is the faster place; off, the
 * gradient is stored beside it.
 * Results equal the separate update's to float32 rounding (the same expressions on the same values).  For a layer
 * that is fused, slp_segment_get_grads returns the bias gradient only (a request for dW fails with SLP_ERR_STATE).
 * Drops captured graphs.  Errors: SLP_ERR_ARG (null handle, on < 0). */
int slp_segment_set_fused_update(slp_segment* seg, int on);

/* ---- several segments trained side by side (end of Sec. 2: partitions are independent jobs) ----
 * The last thing a step does is stream every parameter once (the SGD update); where that is faster it runs on a stream of
 * the handle beside the matrix products that are still to come, and the step normally ends by making `stream` wait for it.
 * With overlap on, slp_segment_step (and slp_segment_step_external) returns without that wait, and the update of
 * the first layer moves to the side stream too, at short batches with the product it is part of (but not for layers of fewer than 224
 * tiles of 128x128 weights and those that slp_segment_set_fused_update names: nothing of them is left pending): whatever the caller enqueues next on `stream` -- typically the
 * step of another segment -- runs beside the tail of this one.  Until the handle's next step, every call on the
 * handle that takes a stream first makes that stream wait for the pending updates (whichever stream it is), so calls
 * through this interface see the same values as without overlap (bit for bit); that step waits
 * for each layer's where it needs it.  A caller that reads or frees the
 * parameter or workspace buffers directly must call slp_segment_join first (slp_segment_destroy and slp_segment_bind
 * wait on the host).  No effect on steps that are captured into a graph; a stream that is being captured cannot wait
 * for updates left pending outside the capture: such a call fails with SLP_ERR_STATE.  With overlap on, the weight updates of
 * large layers are also paced (each of their workgroups pauses between tiles, by an amount that grows with the batch), which
 * roughly doubles their duration and keeps their memory traffic from stalling the matrix products beside them; the caller is
 * expected to keep the device busy behind the step, as a loop over segments does.  Turning overlap off waits on
 * the host for pending updates, after which the handle is back to plain stream order.  Off by default.
 * slp_segment_join: makes `stream` wait for updates a previous step left running; a no-op when none are pending. */
int slp_segment_set_overlap(slp_segment* seg, int on);
int slp_segment_join(slp_segment* seg, slp_stream stream);

/* ---- the joined network at inference (Sec. 2: the partitions can be joined after training; Sec. 4 reports the
 * joined network's test accuracy) and the epoch figures of the training curves ----------------------------
 * slp_count_correct: number of rows n of logits[batch][classes] (dense, row-major, dtype dt, device) whose arg-max
 * column -- the lowest index among equal maxima -- equals targets[n] (int32, device; an id outside [0, classes) never
 * matches).  Logits must not be NaN.  The count goes to *correct_out (int64, device): written when accumulate is 0,
 * added to when it is not (so a loop over the batches of a dataset ends with the dataset's count).  scratch: device
 * memory of at least 4 * ceil(batch / 4) bytes, 4-byte aligned, caller-owned, overwritten (per-block partial counts;
 * they are summed in a fixed order, no atomics).  Asynchronous on `stream`.
 * Errors: SLP_ERR_ARG (null pointer, batch or classes <= 0, unknown dtype), SLP_ERR_ALLOC (scratch too small or
 * misaligned), SLP_ERR_DEVICE.
 * slp_mean_loss: *mean_out = (1/n) sum of losses[0..n) (float32, device; summed in float64 in a fixed order): the
 * epoch mean of the per-step losses that slp_segment_step wrote.  Errors: SLP_ERR_ARG (null, n <= 0), SLP_ERR_DEVICE. */
int slp_count_correct(const void* logits /*device*/, const int32_t* targets /*device*/, int batch, int classes, int dt,
                      void* scratch /*device*/, size_t scratch_bytes, int accumulate, int64_t* correct_out /*device*/,
                      slp_stream stream);
int slp_mean_loss(const float* losses /*device*/, int n, float* mean_out /*device*/, slp_stream stream);

/* slp_count_correct for callers that cannot allocate or hand over scratch memory: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same result as slp_count_correct, bit for bit; the per-block
 * partial counts live in a 64 KiB array inside the library's code object (one copy per GPU the library runs on, held
 * until the process ends) instead of caller memory, and the call allocates nothing and frees nothing.
 * Limit: batch <= SLP_COUNT_STATIC_MAX_BATCH (65536 rows), else SLP_ERR_SHAPE.  Every call on a GPU uses that GPU's one
 * array (each call overwrites the entries it reads; nothing has to be cleared): calls that overlap in time on the
 * same GPU -- different streams, or different host threads -- race and must be serialised by the caller; calls that
 * follow each other on one stream are safe.  Other errors as for slp_count_correct. */
#define SLP_COUNT_STATIC_MAX_BATCH 65536
int slp_count_correct_static(const void* logits /*device*/, const int32_t* targets /*device*/, int batch, int classes,
                             int dt, int accumulate, int64_t* correct_out /*device*/, slp_stream stream);

/* ---- segments in 8 bits ----------------------------------------------------------------
 * Products of 8-bit matrices run at twice the bf16 rate and read half the bytes.  An 8-bit matrix here is two device buffers:
 *   q       [rows][ldq]   e4m3 values (OCP: 4 exponent and 3 fraction bits, largest 448, no infinity), one byte each; q on a 16-byte boundary,
 *                         ldq a multiple of 16; the bytes from the last column up to the next multiple of 16 are read with
 *                         it but not interpreted (so the matrix may be the first columns of a wider one), and written as zeros;
 *   scales  [rows / block, rounded up][lds]   one byte e for each 128 consecutive columns (and, block = 128, each 128 rows): the values
 *                         stand for q * 2^(e - 127); 255 is NaN.  On a 4-byte boundary, lds a multiple of 4 and at least the number of
 *                         blocks of a row; bytes past that number are not interpreted.
 * block is 1 (activations and gradients: a scale for each 128 elements of a row) or 128 (weights: one for each 128 x 128 block, which the
 * transposed matrix shares).  Scales are powers of two because the matrix instruction applies those by itself.  Quantising picks the least
 * power of two, not below 2^-127, under which the block's largest magnitude fits 448, and rounds to nearest even: nothing saturates.  A block
 * that holds an infinity or a NaN gets the scale 255, so that whatever is computed from it is NaN.
 * Rows that are not a multiple of 4096 bytes apart are read faster (fewer of them share a memory channel).
 * The calls take the leading dimensions of every matrix in elements, 64 bits wide; float32 and bf16 matrices may start at any element.  An
 * empty matrix (0 rows) is a call without effect but for sums over its rows, which become zeros.  Common errors: SLP_ERR_ARG (null pointer, negative size, unknown dtype or block),
 * SLP_ERR_SHAPE (a leading dimension below the row, rows or columns above 2^24, more than 2^34 elements, an 8-bit row above 2^22 bytes), SLP_ERR_ALLOC (alignment, workspace),
 * SLP_ERR_DEVICE. */

/* Matrix x[rows][cols] (dtype dt, device) to 8 bits: row-major to q and scales (both or neither null), transposed to qt[cols][ldqt] and
 * scales_t with the rows of x as its columns (both or neither null; at least one of the two layouts).  A transposed copy with block = 1
 * has scales of its own, one for each 128 rows of x; with block = 128 it holds the same values and scales as the row-major one.
 * mask (dtype dt, may be NULL): elements whose mask is not > 0 count as zero -- the ReLU's derivative from its output.  column_sums (float32
 * [cols], may be NULL): the sums of the (masked) columns, the bias's gradient, added in a fixed order; needs workspace. */
size_t slp_quantize_workspace_bytes(int rows, int cols);
int slp_quantize(const void* x /*device*/, int64_t ldx, const void* mask /*device, may be NULL*/, int64_t ldmask, int dt, int rows, int cols, int block,
                 void* q, int64_t ldq, void* scales, int64_t lds, void* qt, int64_t ldqt, void* scales_t, int64_t ldst,
                 float* column_sums /*device, may be NULL*/, void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);

/* out[M][N] = act(A B^T + bias): A [M][K] and B [N][K] 8-bit matrices, each with its own block; bias float32 [N] or NULL; act the ReLU
 * where relu is not 0 (a NaN stays one); out of dtype dt.  Where dt is SLP_F32, or SLP_BF16 | SLP_FLOAT32_SUMS, exact products are added in
 * float32, each matrix's values rounded to bf16 first: that loses nothing between 2^-126 and 1.75 * 2^127, where scales from 2^-117 to 2^119 keep all of them; a larger
 * value counts as infinite, a smaller one loses bits and is zero below 2^-133.  Where it is SLP_BF16 the matrix instruction of 8-bit values adds them, at twice the rate: of each 8 consecutive k it cuts the products off
 * 2^-13 below 2 to the sum of the largest one's exponents, and adds what is left with 24 bits.  At most 7 * 2^-13 of the largest product of each 8 is lost: some 2e-5 of the
 * result where nothing cancels, a hundredth of what rounding it to bf16 costs, but all of a result that small beside products that cancel.  Its scales may be any.  Products of few rows (at most 32) are
 * added in float32 in any case, so that a row alone and in a batch may differ by that much.  Forward: A the input, B the weights.  Gradient of the input:
 * A the gradient of the output, B the transposed weights.  Gradient of the weights: A and B the transposed gradient and input.
 * K = 0 leaves act(bias).  The workspace holds partial products of a contraction that is split over the chip; 256-byte aligned, its size is
 * 0 for most large products. */
#define SLP_FLOAT32_SUMS 16       /* added to slp_product's dt */
size_t slp_product_workspace_bytes(int M, int N, int K);
int slp_product(const void* a /*device*/, int64_t lda, const void* a_scales, int64_t ldsa, int a_block, const void* b, int64_t ldb,
                const void* b_scales, int64_t ldsb, int b_block, const float* bias /*device, may be NULL*/, int relu, int M, int N, int K,
                void* out /*device*/, int64_t ldo, int dt, void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);

/* ---- 8-bit integers with a scale for each row ----
 * A matrix of integers is q [rows][ldq] (signed bytes, alignment and reading past the last column as for 8-bit matrices above) and float32 scales [rows], one for a token of the
 * activations, one for an output channel of the weights: the values are q * scale.
 * slp_quantize_integers: q = round(127 x / max|x|) over each row, ties to even, of the real quotient; scale = max|x| / 127.  A row of zeros has the scale 0, one that holds an
 * infinity or a NaN zeros and the scale NaN.  Written up to the next multiple of 16 columns.
 * slp_product_integers: out[M][N] = act(a_scales[m] b_scales[n] sum over k of A[m][k] B[n][k] + bias[n]), out of dtype dt; the sums are exact, K up to 131071 (any signed byte may stand
 * in A and B); scales, bias and ReLU (where relu is not 0; a NaN stays one) in float32, of which no step on the way leaves the range where the result does not.  The workspace holds parts of a contraction that is split over the chip; 256-byte aligned, 0 for most large products, and no other call's that may run at the same time.
 * Limits and errors as for 8-bit matrices; SLP_ERR_SHAPE also for a longer contraction. */
int slp_quantize_integers(const void* x /*device*/, int64_t ldx, int dt, int rows, int cols, void* q /*device*/, int64_t ldq, float* scales /*device*/, slp_stream stream);
size_t slp_product_integers_workspace_bytes(int M, int N, int K);
int slp_product_integers(const void* a /*device*/, int64_t lda, const float* a_scales, const void* b /*device*/, int64_t ldb, const float* b_scales, const float* bias /*device, may be NULL*/,
                         int relu, int M, int N, int K, void* out /*device*/, int64_t ldo, int dt, void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);

/* Root-mean-square norm of x + residual:
 *   h = x + residual (added in float32, rounded to dt; h = x where residual is NULL);  n = 1 / sqrt(mean over the row of h^2 + eps);  y = h n gamma
 * x, residual, h, y: [rows][dim] of dtype dt; gamma float32 [dim], NULL for ones; rstd float32 [rows] receives n.  h must be given where
 * residual is, and may be x or residual; y, rstd and the 8-bit output (q and scales together, block 1) may be NULL.  The norm and the 8-bit values
 * are of h as stored.  The squares are float32: a row that holds a value beyond 1.8e19 has an infinite mean, n = 0; with eps = 0 a row of zeros, or below 1e-23, has n infinite. */
int slp_rmsnorm(const void* x /*device*/, int64_t ldx, const void* residual /*device, may be NULL*/, int64_t ldr, const float* gamma, float eps, int dt,
                int rows, int dim, void* h, int64_t ldh, void* y, int64_t ldy, void* q, int64_t ldq, void* scales, int64_t lds, float* rstd, slp_stream stream);

/* Its backward pass, from dy (the gradient of y; rounding to 8 bits passes it on), h and rstd as the forward call left them and dh, the gradient that reaches h past
 * the norm (NULL: none):  dx_j = dh_j + n (gamma_j dy_j - h_j n^2 mean over the row of gamma dy h), the gradient of x and of the residual alike;
 * dgamma_j (float32, may be NULL) = sum over the rows of dy_j h_j n, added in a fixed order.  dx may be dy or dh.  Workspace: 256-byte aligned. */
size_t slp_rmsnorm_backward_workspace_bytes(int rows, int dim);
int slp_rmsnorm_backward(const void* dy /*device*/, int64_t lddy, const void* h, int64_t ldh, const float* gamma, const float* rstd, const void* dh, int64_t lddh, int dt,
                         int rows, int dim, void* dx, int64_t lddx, float* dgamma, void* workspace, size_t workspace_bytes, slp_stream stream);

/* ---- the norm of all gradients together ---------------------------------------------------------------
 * tensors[i] (device) holds counts[i] contiguous elements of dtype dts[i]; the three arrays are host memory and are not kept.
 * slp_gradient_norm: *norm_out = sqrt of the sum of all squares (float32; squares and sums are float64, in a fixed order).
 * slp_clip_gradients: out[i] = c tensors[i] with c = min(1, max_norm / (norm + 1e-6)); out[i] may be tensors[i] (out NULL: all of them), where c = 1 costs
 * nothing.  A norm that is not finite (in float32, as norm_out holds it) leaves the values as they are: look at *norm_out and skip the update.  norm_out may be NULL.
 * Workspace: 256-byte aligned.  Errors: SLP_ERR_ARG (null array or tensor, negative count, unknown dtype, max_norm not > 0), SLP_ERR_ALLOC, SLP_ERR_DEVICE. */
size_t slp_gradient_norm_workspace_bytes(int n);
int slp_gradient_norm(const void* const* tensors /*host*/, const int64_t* counts /*host*/, const int* dts /*host*/, int n, float* norm_out /*device*/,
                      void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);
int slp_clip_gradients(const void* const* tensors /*host*/, void* const* out /*host, may be NULL*/, const int64_t* counts /*host*/, const int* dts /*host*/, int n,
                       float max_norm, float* norm_out /*device, may be NULL*/, void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);

/* ---- losses over the classes of a linear layer --------------------------------------------------
 * z = x W^T + b for rows x[rows][dim] and weights w[classes][dim] (both of dtype dt), bias float32 [classes] or NULL.  The logits z are computed tile by tile and do not have to
 * fit in memory.  Beside its operands and outputs a call takes a workspace of, at most,
 *   1 GiB for logits that are kept in float32 until their gradient is due (the others are computed again; none where no gradient is wanted), 256 MB for the gradient of a piece of the
 *   classes, or 256 classes of every row where that is more (1 GiB for 2^20 rows in float32); rows of both are padded by up to 256 bytes;
 *   x once more for dw, or where it cannot be read in place, and up to 2 GiB of w where that cannot, their rows padded as well;
 *   partial sums: 68 MB, or float32 [rows][dim] where that is more, for dx, 68 MB for dw, 20 MB for dbias, 64 MB for logits of few tiles;
 *   8 bytes for each row and 16 classes (and 64 of these a row), for each class (dbias of a distillation) and for each entry of a row, 32 for each row, 4 KB.
 * For each row
 *   lse = log sum over the classes of exp(z / T)                                      (float32 [rows], of rows that do not count as well)
 * slp_linear_cross_entropy (T = 1): targets[rows] are class ids (target_bytes 4 or 8: int32 or int64).  loss = lse - z_target.
 * slp_linear_distillation: top[rows][k] (dtype top_dt) are a teacher's logits of the classes top_classes[rows][k] (class_bytes 4 or 8), in any order, k from 1 to 1024,
 *   p = softmax(top / T) over the row's entries, loss = T^2 sum of p (log p - log softmax(z / T) at the entry's class).  A class may stand in several entries of a row, whose probabilities
 *   then add up in the gradient.  0.001 <= T <= 1000.
 * An id outside [0, classes) is no class: the row of a cross-entropy, the entry of a distillation does not count (padding), nor does an entry whose top is -infinity.  A row
 * without an entry that counts has the loss 0, does not enter the mean, and its x reaches no output but its own lse, whatever it holds.
 * *loss = the mean of losses[rows] over the rows that count, 0 where none does.  The gradients, each wanted where its pointer is not NULL, are those of scale * *loss:
 *   dz = scale T (softmax(z / T) - p) / (rows that count);  dx[rows][dim] = dz W, of dtype dt;  dw[classes][dim] = dz^T x, of dtype dw_dt;  dbias (float32 [classes]) = sums of dz
 * Products add in float32; dz over its common factor is rounded to dt where it enters the products for dx and dw, not for dbias.  Float32 operands are multiplied to 2^-24 as float32 arithmetic
 * does; above 3.39e38 they count as infinite, below 2^-102 they lose bits, and a product with an infinity is NaN.  Sums are in a fixed order, targets' in integers: the same bits every time.
 * Logits that are NaN or +infinity make their row's loss, and what it reaches, NaN; -infinity (a class that the bias masks out) is a probability of 0.
 * Matrices may start at any element; x and w whose rows start on 16-byte boundaries and whose dim fills them are read in place, others are copied to the workspace first.  Outputs must not overlap
 * operands.  No rows: a loss of 0, dw and dbias become zeros.  The workspace is 256-byte aligned, of slp_linear_loss_workspace_bytes for the same pointers and sizes (0 for those that the calls refuse), and of no other call that may run at the same time; top: k of a distillation, 0 for a
 * cross-entropy; outputs: SLP_LOSS_* of the gradients wanted.
 * Errors: SLP_ERR_ARG (null pointer, negative rows, no classes or dim, unknown dtype or id size, k, T or scale out of range), SLP_ERR_SHAPE (a leading dimension below the row or, of x and w, above 2^20;
 * more than 2^20 rows or dim, 2^24 classes, 2^33 elements of x or w, 2^36 logits, 2^25 targets; with dw, rows of x that come to 2 GiB), SLP_ERR_ALLOC (alignment, workspace), SLP_ERR_DEVICE. */
enum { SLP_LOSS_DX = 1, SLP_LOSS_DW = 2, SLP_LOSS_DBIAS = 4 };
size_t slp_linear_loss_workspace_bytes(const void* x, int64_t ldx, const void* w, int64_t ldw, int dt, int rows, int classes, int dim, int top, int outputs);
int slp_linear_cross_entropy(const void* x /*device*/, int64_t ldx, const void* w /*device*/, int64_t ldw, const float* bias /*device, may be NULL*/, int dt, int rows, int classes, int dim,
                             const void* targets /*device*/, int target_bytes, float scale, float* loss /*device*/, float* losses /*device*/, float* lse /*device*/, void* dx, int64_t lddx,
                             void* dw, int64_t lddw, int dw_dt, float* dbias, void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);
int slp_linear_distillation(const void* x /*device*/, int64_t ldx, const void* w /*device*/, int64_t ldw, const float* bias /*device, may be NULL*/, int dt, int rows, int classes, int dim,
                            const void* top /*device*/, int64_t ldtop, int top_dt, const void* top_classes /*device*/, int64_t ldclasses, int class_bytes, int k, float temperature,
                            float scale, float* loss /*device*/, float* losses /*device*/, float* lse /*device*/, void* dx, int64_t lddx, void* dw, int64_t lddw, int dw_dt, float* dbias,
                            void* workspace /*device*/, size_t workspace_bytes, slp_stream stream);

/* ---- measurement hooks -------------------------------------------------------------
 * When enabled, every matrix-product launch of the segment is bracketed by HIP
 * events on its stream.  slp_segment_profile_read synchronises the recorded events,
 * returns the accumulated device time of those launches (milliseconds), their count
 * and their algorithmic FLOPs (2*M*N*K with unpadded sizes), then clears the log.
 * on > 1 additionally creates `on` event pairs up front so that none has to be
 * created between timed launches. */
int slp_segment_profile_enable(slp_segment* seg, int on);
int slp_segment_profile_read(slp_segment* seg, double* gemm_ms, int64_t* gemm_launches, double* gemm_flops);

/* Sustained matrix-pipe rate of the device the caller has made current: a register-only
 * loop of the MFMA instructions the matrix products use (bf16 16x16x32 or float32
 * 32x32x2, 8 wavefronts per compute unit, one workgroup per compute unit, pseudo-random
 * operands), `iters` iterations of 16 MFMA groups per wavefront, timed with HIP events
 * on `stream` after a short warm-up launch.  Synchronous.  It is the rate the chip holds
 * under its power limit with no memory traffic at all: the practical ceiling to read a
 * measured matrix-product rate against, beside the published peak.
 * scratch: device buffer of at least 2048 bytes per compute unit (caller-owned, overwritten).
 * tflops_out (host) receives the rate in TFLOP/s, ms_out (host, may be NULL) the duration.
 * Errors: SLP_ERR_ARG (dtype, iters outside [1, 2^24], null pointers), SLP_ERR_SHAPE
 * (scratch too small), SLP_ERR_DEVICE. */
int slp_probe_mfma_rate(int dtype, int iters, void* scratch /*device*/, size_t scratch_bytes, double* tflops_out /*host*/,
                        double* ms_out /*host, may be NULL*/, slp_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* SLP_H */
