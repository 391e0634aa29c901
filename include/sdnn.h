/*
 * sdnn.h -- C ABI of the MI355X Sparse DNN inference library (libsdnn.so).
 *
 * Computes the Sparse DNN Challenge inference of Kepner et al. (2019):
 *   Sec. II, batched inference equation:  Y_{l+1} = h(Y_l W_l + B_l), with h(y) = min(YMAX, max(y, 0))
 *   (ReLU with the challenge's upper limit, Sec. II; YMAX = 32 in the Sec. V listing), the bias added
 *   only where Y_l W_l is nonzero (the Sec. V serial loop), for every layer l = 0..L-1;
 *   then the categories: the rows of the final Y with any entry > 0 (Sec. V, second timed step).
 *
 * Numerics: fp32. Every output is z = fma(y_{k_m}, w_m, ... fma(y_{k_0}, w_0, +0)) over the sources of
 * its column in ascending source order, one rounding per term; then t = z + b (one fp32 add) and
 * y = (z != 0) ? min(ymax, max(0, t)) : 0, with zeros written as +0. Results are therefore identical
 * on every run and match a sequential fp32 evaluation in that order bit for bit.
 *
 * Call order (Sec. V: download, load, set bias untimed; evaluate all layers and identify categories
 * timed; compare untimed):
 *   sdnn_create -> sdnn_load_layers (any chunks covering layers 0..L-1) -> [sdnn_infer ->
 *   sdnn_categories]* -> diagnostics -> sdnn_destroy.
 * The timed region of the challenge is sdnn_infer + sdnn_categories.
 *
 * Ownership: the library owns the handle and its device copies of the weights and biases. The caller
 * owns the input activations, the workspace, the stream and every host array; host arrays may be
 * reused as soon as a call returns. No call after sdnn_load_layers allocates device memory.
 *
 * Errors: no exception crosses the ABI. Every call returns an sdnn_status; sdnn_last_error() gives a
 * thread-local message for the last failure. SDNN_EINVAL, SDNN_ESTATE and SDNN_ERANGE leave the
 * handle unchanged. SDNN_EDEVICE (a HIP call failed) poisons the handle: every later call except
 * sdnn_destroy returns SDNN_EDEVICE.
 *
 * A handle is not thread-safe; use one handle per thread.
 */
#ifndef SDNN_H
#define SDNN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sdnn_net sdnn_net;

typedef enum {
  SDNN_OK = 0,
  SDNN_EINVAL = 1,  /* an argument is malformed or out of range */
  SDNN_ENOMEM = 2,  /* an allocation failed: of device memory (only sdnn_load_layers) or of host memory */
  SDNN_EDEVICE = 3, /* a HIP call failed; the handle is poisoned */
  SDNN_ESTATE = 4,  /* call out of order (e.g. infer before every layer is loaded) */
  SDNN_ERANGE = 5   /* output capacity too small; the needed size is reported */
} sdnn_status;

/* Create a network of n_layers layers of n_neurons neurons each (Sec. II: N neurons per layer,
 * L layers). ymax is the upper limit of h (Sec. II; 32 in the challenge) and must be finite and > 0.
 * 1 <= n_neurons <= 65536, 1 <= n_layers <= 1000000. Host-only: touches no device. */
sdnn_status sdnn_create(sdnn_net **out, int32_t n_neurons, int32_t n_layers, float ymax);

/* Opt in (enable = 1) to kernels that exploit layers whose weights are all equal and whose biases
 * are all equal: such a layer is read as one weight, one bias and 16-bit source lists; layer 0 on
 * binary inputs is computed from counts of active sources; columns that share their source list are
 * computed once. Results are bit-identical to the default. Off by default, because the paper's
 * Sec. V lists exploiting the repetitive structure of weight and bias values among the things a
 * challenge submission should avoid: by default every layer reads each edge's weight and each
 * neuron's bias from memory. Host-only. Must precede the first sdnn_load_layers (SDNN_ESTATE
 * afterwards); enable other than 0 or 1 is SDNN_EINVAL. */
sdnn_status sdnn_enable_equal_value_kernels(sdnn_net *net, int32_t enable);

/* Load layers [l0, l0 + nl) (Sec. V: load the DNN; create the bias vectors b_l).
 * Weights in CSC, one column per output neuron j (Sec. II: W(i, j) != 0 connects neuron i to
 * neuron j, and rows y multiply W from the left, so column j lists the inputs of neuron j):
 *   col_ptr: nl * (n_neurons + 1) int64, host. Layer i's column j holds entries
 *            [col_ptr[i*(N+1) + j], col_ptr[i*(N+1) + j + 1]) of row_idx/val. Offsets are absolute
 *            indexes into row_idx/val, non-decreasing within a layer; layer i starts where layer i-1
 *            ends (col_ptr[i*(N+1)] == col_ptr[(i-1)*(N+1) + N]); col_ptr[0] may be nonzero.
 *   row_idx: int32 source neurons, in [0, N), strictly ascending within each column, host.
 *   val:     fp32 weights, finite, host.
 *   bias:    nl * n_neurons fp32, finite, host; bias[i*N + j] = b_l(j) for l = l0 + i.
 * A column may hold at most 4096 sources. Each layer may be loaded once. The call copies the data
 * into device memory it owns (allocated here, on the current device) and packs it into the layout
 * the kernels read; it synchronizes `hip_stream` (a hipStream_t, or NULL for the default stream)
 * before returning. With sdnn_enable_equal_value_kernels on, columns of a one-weight layer with 32
 * sources that share their source list (and so their output) are computed once when the next layer
 * is loaded right after it, in the same call or the next one; loading layers in ascending order
 * therefore never costs speed, and any order gives the same results. The first call on a handle
 * also creates the host-side objects the timed calls use (read-back events, pinned host words), so
 * that sdnn_infer and sdnn_categories allocate nothing. */
sdnn_status sdnn_load_layers(sdnn_net *net, int32_t l0, int32_t nl, const int64_t *col_ptr,
                             const int32_t *row_idx, const float *val, const float *bias,
                             void *hip_stream);

/* Bytes of device workspace sdnn_infer needs for n_rows input rows (activation buffers, live-row
 * lists, flags, counters). n_rows >= 0. Returns 0 for a NULL handle or negative n_rows. */
size_t sdnn_workspace_bytes(const sdnn_net *net, int64_t n_rows);

/* TIMED. Evaluate all layers (Sec. II batched equation) for the n_rows input rows in y0.
 *   y0:        device pointer, n_rows x n_neurons fp32, row-major (Sec. IV: one flattened input per
 *              row), finite; read-only, so the same y0 can be run again. Not needed after the call's
 *              work completes on the stream.
 *   workspace: device pointer, >= sdnn_workspace_bytes(net, n_rows) bytes, 256-byte aligned; owned
 *              by the caller, overwritten, must stay untouched until sdnn_categories returns and
 *              while diagnostics are read.
 *   hip_stream: hipStream_t (NULL = default stream) on which all work is enqueued; not one that is
 *              being captured into a graph (SDNN_ESTATE for n_rows > 0, nothing is enqueued).
 * Rows that become all zero are dropped from later layers: their activations stay zero for every W
 * and b, since Z = 0 gets no bias. The call enqueues layers in chunks and reads the live-row count
 * back from the device every few layers, so it may block until earlier layers finish; once no row
 * is live it stops enqueuing. Requires every layer to be loaded (SDNN_ESTATE otherwise). */
sdnn_status sdnn_infer(sdnn_net *net, const float *y0, int64_t n_rows, void *workspace,
                       size_t workspace_bytes, void *hip_stream);

/* TIMED. sdnn_infer for callers that cannot allocate device memory (tight serving
 * loops, harnesses that forbid allocation): the same computation and results,
 * with the workspace taken from a 64 MiB array in the library's device memory instead of a caller
 * buffer. Allocates nothing (no hipMalloc, hipFree or allocating library call). The array is one per
 * device, shared by every handle and call on that device, and keeps the last call's contents: calls
 * that overlap on one device race, so serialize them (one stream, or wait for sdnn_categories) and
 * read a run's diagnostics (sdnn_live_counts, sdnn_final_rows) before the next static run on that
 * device. n_rows must satisfy sdnn_workspace_bytes(net, n_rows) <= 64 MiB; larger batches return
 * SDNN_ERANGE (nothing is enqueued). Other arguments and errors as for sdnn_infer. */
sdnn_status sdnn_infer_static(sdnn_net *net, const float *y0, int64_t n_rows, void *hip_stream);

/* TIMED. Wait for the last sdnn_infer and report its categories (Sec. V: the rows of the final
 * matrix with entries > 0): 0-based row indexes into y0, ascending, written to ids (host,
 * capacity entries). *count receives the number of categories. ids == NULL or capacity < count
 * returns SDNN_ERANGE with *count set (query mode). SDNN_ESTATE before any sdnn_infer. */
sdnn_status sdnn_categories(sdnn_net *net, int64_t *ids, int64_t capacity, int64_t *count);

/* Diagnostics (untimed). Live-row counts of the last sdnn_infer: counts[0] = input rows with any
 * nonzero entry, counts[l] = rows with any entry > 0 after layer l-1, for l = 1..n_layers (zeros
 * after the layer where no row was left). counts: host, n_layers + 1 entries. */
sdnn_status sdnn_live_counts(sdnn_net *net, int64_t *counts);

/* Diagnostics (untimed). Final activations of rows ids[0..n) (0-based, < n_rows of the last
 * sdnn_infer) into out_host (n x n_neurons fp32, row-major); rows that are not categories are all
 * zero. SDNN_EINVAL for an id out of range. */
sdnn_status sdnn_final_rows(sdnn_net *net, const int64_t *ids, int64_t n, float *out_host);

/* Diagnostics. enable == 1: every later sdnn_infer records a HIP event pair on its stream around
 * each layer's kernels (the layer SpMM with its fused epilogue; not the compaction), and
 * sdnn_categories adds the elapsed times to per-layer totals. enable == 2: the same for large
 * layers only (layers whose live rows take more than one round of tiles, or, for widths staged in
 * LDS, while more than 256 rows may be live), so that the event records do not slow the long tail
 * of layers with few rows. enable == 0 stops recording; other values are SDNN_EINVAL.
 * Creates its events here (needs the device); enabling again resets the totals. */
sdnn_status sdnn_set_profiling(sdnn_net *net, int32_t enable);

/* Diagnostics. Per-layer totals since profiling was enabled: ms[l] milliseconds over runs[l] timed
 * runs of layer l (0 for layers not recorded). ms, runs: host arrays of n_layers entries. */
sdnn_status sdnn_layer_times(sdnn_net *net, double *ms, int64_t *runs);

/* Kernel families reported by sdnn_layer_info. */
typedef enum {
  SDNN_KERNEL_NONE = 0,                 /* layer not run (every row had died) */
  SDNN_KERNEL_LDS_TILE = 1,             /* activation tiles staged in LDS (k_layer_lds, k_layer_lds32) */
  SDNN_KERNEL_GLOBAL_TILE = 2,          /* fp32 activations in global memory: feature-major tiles (k_layer_gfm) or,
                                           up to 16384 neurons, rows (k_layer_seg) */
  SDNN_KERNEL_GLOBAL_TILE_CODES = 3,    /* one-byte dictionary codes of the inputs (k_layer_gfm_u8) */
  SDNN_KERNEL_GLOBAL_TILE_FEW_ROWS = 4, /* at most 8 tiles, whole chains in flight (k_layer_gfm_small) */
  SDNN_KERNEL_BITS = 5,                 /* layer 0 from bit-packed binary inputs (k_pack_bits, k_layer_bits) */
  SDNN_KERNEL_BITS_TO_CODES = 6,        /* the same, writing one-byte dictionary codes */
  SDNN_KERNEL_BITS_COUNT = 7,           /* layer 0 of a uniform layer on binary inputs, by bit-sliced counts
                                           (k_pack_bits, k_count_dict, k_layer_count); only with
                                           sdnn_enable_equal_value_kernels */
  SDNN_KERNEL_LDS_FUSED = 8,            /* every layer from this one on, in one launch that keeps each
                                           workgroup's rows in LDS (k_layers_lds, k_layers_lds32); it is counted
                                           at its first layer, later layers report 0 launches */
  SDNN_KERNEL_GLOBAL_TILE_CODES16 = 9   /* two-byte dictionary codes of the inputs, for inputs of 257 to
                                           4096 distinct values (k_layer_gfm_u8 on 16-bit codes) */
} sdnn_kernel_kind;

/* Diagnostics (untimed). For each layer of the last sdnn_infer: the kernel family that ran it
 * (sdnn_kernel_kind) and its number of kernel launches, those that encoded its inputs included (for
 * layers timed with events, the event pair spans these launches). kernel, launches: host arrays of
 * n_layers entries. */
sdnn_status sdnn_layer_info(sdnn_net *net, int32_t *kernel, int32_t *launches);

/* Diagnostics (untimed). The name of the kernel that ran `layer` of the last sdnn_infer, for families of more than
 * one kernel the one it was: "k_layer_lds" or "k_layer_lds32" (SDNN_KERNEL_LDS_TILE), "k_layers_lds" or
 * "k_layers_lds32" (SDNN_KERNEL_LDS_FUSED), "k_layer_gfm" or "k_layer_seg" (SDNN_KERNEL_GLOBAL_TILE);
 * two kernels are joined by '+'. *name receives a string that is never freed. */
sdnn_status sdnn_layer_kernel(sdnn_net *net, int32_t layer, const char **name);

/* Free the handle and its device memory. NULL is a no-op. */
void sdnn_destroy(sdnn_net *net);

/* Thread-local description of the last failed call ("" if none). */
const char *sdnn_last_error(void);

/* Which kernel family the handle uses for its width: 0 = activation tiles staged in LDS,
 * 1 = tiles gathered from global memory (widths too large for LDS). -1 for NULL. */
int32_t sdnn_kernel_path(const sdnn_net *net);

/* ---------------------------------------------------------------------------------------------------------------
 * The dense readout: a layer of n_classes outputs on rows of n_features values, such as a network's final rows
 * (sdnn_final_rows leaves them on the host; they are uploaded for these calls). These calls need no handle. All
 * matrices are row-major in device memory; a stride is the distance of two rows in values and at least the row's
 * length. Everything is enqueued on hip_stream (NULL = default stream), of the current device, on which all pointers
 * must be usable; no call waits, allocates or keeps anything, so each can be captured into a graph. A workspace is the
 * caller's, 256-byte aligned, overwritten, and must stay untouched until the call's work completes on the stream;
 * SDNN_ERANGE where it is too small. Malformed arguments are SDNN_EINVAL and enqueue nothing. SDNN_EDEVICE: a launch
 * failed (some of the call's work may have been enqueued). Results do not depend on what else runs: the same inputs
 * give the same bits. */

typedef enum {
  SDNN_FP32 = 0,
  SDNN_BF16 = 1
} sdnn_dtype;

/* Bytes of workspace for sdnn_readout_loss (gradient = 0) or for both calls (gradient = 1). It grows with
 * n_rows * n_features and n_features * n_classes (fp32 operands are held in 16-bit parts, unaligned ones are
 * copied). What it holds for each row and class together is bounded however many there are of both: for the loss by 256
 * MB (or up to 64 fp32 parts of at most 2^24 logits, where rows are long), for the gradient by 6 bytes times the larger of
 * 2^26 and 256 n_rows as well. 0 for sizes that the calls refuse: n_rows in [0, 2^24],
 * n_classes in [1, 2^24], n_features in [1, 2^20]. */
size_t sdnn_readout_workspace_bytes(int64_t n_rows, int64_t n_classes, int64_t n_features, int32_t dtype,
                                    int32_t gradient);

/* Softmax cross entropy of the logits l = x w^T, which are not kept (where there are at most 2^24 of
 * them, sums of parts of them may pass through the workspace).
 *   x: n_rows x n_features, w: n_classes x n_features, both of `dtype`, row strides ldx and ldw.
 *   labels: n_rows int64. A label outside [0, n_classes) leaves its row out: its loss is 0.
 *   loss: n_rows fp32, lse_t - l_{t, label}.  lse: n_rows fp32 (or NULL), log sum_v exp l_tv, also of rows
 *   that are left out; sdnn_readout_grad needs it.
 * Sums are fp32, of exact products for bf16 inputs; fp32 inputs are multiplied as they are or as two fp16 parts each
 * (22 bits or more of each value down to 2^-17 of its row's largest). A row that holds an infinity or a NaN has a NaN
 * loss. */
sdnn_status sdnn_readout_loss(const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t dtype,
                              const int64_t *labels, int64_t n_rows, int64_t n_classes, int64_t n_features,
                              float *loss, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/* The gradient of sum_t row_grad_t loss_t, or, with row_grad == NULL, of the mean loss over the rows with a label:
 *   G_tv = row_grad_t (exp(l_tv - lse_t) - [v = label_t]),  dx = G w,  dw = G^T x.
 *   lse: as sdnn_readout_loss left it for these x and w, of whose logits exp(l - lse) takes the same bits. row_grad:
 *   n_rows fp32 or NULL.
 *   dx: n_rows x n_features, dw: n_classes x n_features, of `dtype`, row strides lddx and lddw; overwritten. Either
 *   may be NULL: not computed. Neither may overlap an input.
 * Rows without a label add nothing to dw and have a dx of zeros, whatever x, lse and row_grad hold there. For bf16 G is
 * rounded to bf16 once (as a fraction of the largest row_grad), between two fp32 sums. For fp32 inputs the logits are
 * the loss's, and G, w and x are multiplied as they are or as three bf16 parts each (all 24 bits of a value down to 2^-110),
 * so that values of very different sizes keep what fp32 keeps of them. */
sdnn_status sdnn_readout_grad(const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t dtype,
                              const int64_t *labels, const float *lse, const float *row_grad, int64_t n_rows,
                              int64_t n_classes, int64_t n_features, void *dx, int64_t lddx, void *dw, int64_t lddw,
                              void *workspace, size_t workspace_bytes, void *hip_stream);

/* Bytes of workspace for sdnn_orthogonalize; 0 for sizes that it refuses: batch in [0, 65535], rows and cols in
 * [1, 2^20]. */
size_t sdnn_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols);

/* Orthogonalise `batch` matrices of rows x cols by Newton-Schulz products: X = g / (||g||_F + eps), then `steps`
 * times X <- a X + (b A + c A A) X with A = X X^T and coefficients = {a, b, c} (host, 3 values), in the smaller of the
 * two sizes (for rows > cols the same X is found from X^T X).
 *   g, out: device, of `dtype`, row strides ldg and ldo, batch strides (values; ignored for one matrix). out may be
 *   g itself (same strides), and may not overlap it otherwise.
 * Every product is of factors held in two fp16 parts under one power of two for a matrix (2^-38 of a bound of its entries
 * is the smallest part), with fp32 sums: errors are fp32's against the matrix's norm, a row far smaller than the others
 * keeps fewer bits. The result is rounded to `dtype` once. A
 * matrix of zeros gives zeros (eps > 0); one with an infinity or a NaN gives NaN where those reach.
 * steps in [0, 32]; eps >= 0; |coefficients| <= 1e6. */
sdnn_status sdnn_orthogonalize(const void *g, int64_t ldg, int64_t batch_stride_g, void *out, int64_t ldo,
                               int64_t batch_stride_o, int32_t dtype, int64_t batch, int64_t rows, int64_t cols,
                               int32_t steps, const float *coefficients, float eps, void *workspace,
                               size_t workspace_bytes, void *hip_stream);

/* Rows of microscaled 4-bit floats: n_values values are held in sdnn_mx_blocks(n_values) blocks of 32 (whole runs of
 * 4 blocks; 0 for n_values outside [1, 2^20]). A matrix of n_rows rows is
 *   codes:  n_rows x 16 * blocks bytes, 16-byte aligned; a byte holds values 2i (low half) and 2i + 1: a sign bit over a
 *           magnitude code of {0, 0.5, 1, 1.5, 2, 3, 4, 6};
 *   scales: n_rows x blocks bytes, 4-byte aligned; s stands for 2^(s - 127), 255 for a block of NaN.
 * Codes past n_values are zero. */
int64_t sdnn_mx_blocks(int64_t n_values);

/* Quantise x (n_rows x n_values of `dtype`, row stride ldx). A block's scale is 2^(floor(log2 max|x|) - 2), at least
 * 2^-127; values are rounded to the nearest code, ties to the even one, magnitudes over 6 to 6. A block with
 * an infinity or a NaN becomes NaN. */
sdnn_status sdnn_mx_quantize(const void *x, int64_t ldx, int32_t dtype, int64_t n_rows, int64_t n_values, uint8_t *codes,
                             uint8_t *scales, void *hip_stream);

/* The values that codes and scales stand for, in out (n_rows x n_values of `dtype`, row stride ldo). */
sdnn_status sdnn_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t n_rows, int64_t n_values, void *out,
                               int64_t ldo, int32_t dtype, void *hip_stream);

/* out = x w^T of quantised rows (x: n_rows, w: n_outputs rows, both of n_values): fp32 sums of exact products, rounded
 * to `dtype` once. out: n_rows x n_outputs, row stride ldo. */
sdnn_status sdnn_mx_product(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes,
                            const uint8_t *w_scales, int64_t n_rows, int64_t n_outputs, int64_t n_values, void *out,
                            int64_t ldo, int32_t dtype, void *hip_stream);

/* The same for rows x of `dtype` (row stride ldx) that are quantised on the way: a readout's answer with its weights held
 * in 4 bits. The products are those of sdnn_mx_quantize and sdnn_mx_product; for few rows their fp32 sums may be taken
 * in another order. */
size_t sdnn_mx_linear_workspace_bytes(int64_t n_rows, int64_t n_values);
sdnn_status sdnn_mx_linear(const void *x, int64_t ldx, int32_t dtype, const uint8_t *w_codes, const uint8_t *w_scales,
                           int64_t n_rows, int64_t n_outputs, int64_t n_values, void *out, int64_t ldo, void *workspace,
                           size_t workspace_bytes, void *hip_stream);

/* A gated hidden layer, such as one under a readout: h = act(g) * u with g = x w_gate^T and u = x w_up^T. The conventions
 * are the readout's. */
typedef enum {
  SDNN_SILU = 0, /* g / (1 + exp(-g)) */
  SDNN_GELU = 1, /* g times the normal distribution's integral up to g (by the error function) */
  SDNN_RELU = 2  /* max(g, 0); its slope at 0 is 0 */
} sdnn_activation;

/* Bytes of workspace for sdnn_gated (gradient = 0), for both calls where the gradient gets gate and up (1), or where
 * it computes them again (2). 0 for sizes that the calls refuse: n_rows in [0, 2^24], n_hidden in [1, 2^19], n_features in
 * [1, 2^20]. For the gradient it grows with n_rows * n_hidden. */
size_t sdnn_gated_workspace_bytes(int64_t n_rows, int64_t n_hidden, int64_t n_features, int32_t dtype, int32_t gradient);

/* The layer.
 *   x: n_rows x n_features, w_gate, w_up: n_hidden x n_features, all of `dtype`, with their row strides.
 *   h: n_rows x n_hidden of `dtype`, written.  gate, up: the same size, or NULL: g and u, rounded to `dtype`, for
 *   sdnn_gated_grad. None of the three may overlap an input or another.
 * g and u are fp32 sums, of exact products for bf16 inputs; fp32 inputs are multiplied as they are or as two fp16 parts
 * each (22 bits or more of each value down to 2^-17 of its row's largest). h is taken from these sums, whether they are kept or
 * not, and rounded once; for fp32 act keeps its relative precision where it goes to zero. An infinity or a NaN reaches the
 * results of its own row of x or of its own outputs alone; NaN may stand where the formula has an infinity. */
sdnn_status sdnn_gated(const void *x, int64_t ldx, const void *w_gate, int64_t ldw_gate, const void *w_up, int64_t ldw_up,
                       int32_t dtype, int32_t activation, int64_t n_rows, int64_t n_hidden, int64_t n_features, void *h,
                       int64_t ldh, void *gate, int64_t ldgate, void *up, int64_t ldup, void *workspace,
                       size_t workspace_bytes, void *hip_stream);

/* Its gradient: with dg = dh * u * act'(g) and du = dh * act(g),
 *   dx = dg w_gate + du w_up,  dw_gate = dg^T x,  dw_up = du^T x.
 *   gate, up: as sdnn_gated kept them, or both NULL: they are computed again, with the same results.
 *   dh: n_rows x n_hidden.  dx: n_rows x n_features, dw_gate, dw_up: n_hidden x n_features; overwritten. Each may be
 *   NULL: not computed. None may overlap an input or another. All are of `dtype`.
 * For bf16 dg and du are rounded to bf16 once, between fp32 arithmetic and fp32 sums. fp32 values are multiplied as they
 * are or as three bf16 parts each (all 24 bits of a value down to 2^-110). With no rows dw_gate and dw_up are zeros. */
sdnn_status sdnn_gated_grad(const void *x, int64_t ldx, const void *w_gate, int64_t ldw_gate, const void *w_up,
                            int64_t ldw_up, int32_t dtype, int32_t activation, const void *gate, int64_t ldgate,
                            const void *up, int64_t ldup, const void *dh, int64_t lddh, int64_t n_rows, int64_t n_hidden,
                            int64_t n_features, void *dx, int64_t lddx, void *dw_gate, int64_t lddw_gate, void *dw_up,
                            int64_t lddw_up, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Gradients clipped by their common norm. A tensor is a matrix of rows x cols values of `dtype` in device memory, `ld` values
 * from row to row (ignored for one row). */
typedef struct {
  void *data;
  void *out;    /* sdnn_clip: where the scaled values go; NULL or data: to data itself */
  int64_t rows, cols; /* either may be 0 */
  int64_t ld, ldo;    /* ldo: of out; where out is data, the same */
  int32_t dtype;
} sdnn_tensor;

/* Bytes of workspace for a list of n_tensors, whatever their sizes; 0 outside [0, 4096]. */
size_t sdnn_clip_workspace_bytes(int64_t n_tensors);

/* norm (device, one fp32) = the square root of the sum of squares of all values of the tensors (a host array, read
 * during the call). Squares and their sums are fp64. */
sdnn_status sdnn_global_norm(const sdnn_tensor *tensors, int64_t n_tensors, float *norm, void *workspace,
                             size_t workspace_bytes, void *hip_stream);

/* The norm, and every value times min(1, max_norm / norm), a factor in fp32, rounded to the tensor's type once. A norm
 * that is NaN makes NaN of all values, an infinite one zeros, and NaN of what was infinite. Tensors that are written may
 * not overlap each other, nor an input that is not their own; a list that writes two of them to one address is refused.
 * max_norm >= 0. */
sdnn_status sdnn_clip(const sdnn_tensor *tensors, int64_t n_tensors, float max_norm, float *norm, void *workspace,
                      size_t workspace_bytes, void *hip_stream);

/* Weights of 4 bits with a scale for each group of 32, 64 or 128 values of a row: w = scale * (code - 8), or, with offsets,
 * scale * code + offset, code in [0, 15]. A matrix of n_rows rows of n_values values is
 *   codes:   n_rows x groups * group / 2 bytes, 16-byte aligned, groups = sdnn_grouped_groups(n_values, group) (0 for
 *            n_values outside [1, 2^20] and other groups); a byte holds values 2i (low half) and 2i + 1;
 *   scales, offsets: n_rows x groups of `dtype`; offsets may be NULL.
 * Codes past n_values may be anything. `dtype` is also that of the rows that they are multiplied with. */
int64_t sdnn_grouped_groups(int64_t n_values, int32_t group);

/* Quantise w (n_rows x n_values, row stride ldw). Without offsets a group's scale is its largest magnitude over 7; with
 * them (max - min) / 15, and the offset is the minimum. Both are rounded to `dtype` (the scale to the number below where the
 * largest code would stand for an infinity), then codes to the nearest value that they can stand for, ties to the even
 * code. A group with an infinity or a NaN stands for NaN. */
sdnn_status sdnn_grouped_quantize(const void *w, int64_t ldw, int32_t dtype, int64_t n_rows, int64_t n_values,
                                  int32_t group, uint8_t *codes, void *scales, void *offsets, void *hip_stream);

/* The values that they stand for, one fp32 product and sum each, rounded to `dtype`, in out (n_rows x n_values, row stride
 * ldo). */
sdnn_status sdnn_grouped_dequantize(const uint8_t *codes, const void *scales, const void *offsets, int32_t dtype,
                                    int64_t n_rows, int64_t n_values, int32_t group, void *out, int64_t ldo,
                                    void *hip_stream);

/* out (n_rows x n_outputs, row stride ldo) = x w^T for rows x (n_rows x n_values, row stride ldx) and n_outputs rows of codes.
 * Few rows (up to 64; up to 128 of bf16 or 256 of fp32 values where n_outputs is 4096 or more and w holds 2^24 values or
 * more): scales and offsets are multiplied with fp32 sums over their groups, of exact products. For more rows w is rounded
 * to `dtype` first, as sdnn_grouped_dequantize has it, and multiplied with x: exact products for bf16, fp32 values as they
 * are or as two fp16 parts (22 bits or more of each value down to 2^-17 of its row's largest). Sums are fp32, rounded to
 * `dtype` once. An infinity or a NaN in a row of x leaves none of its results finite; a group that stands
 * for NaN makes NaN of its output's. out may not overlap an input.
 * The workspace is 0 bytes for up to 16 rows that a workgroup holds in one piece (16 of 4352 bf16 values, 16 of 1152 fp32
 * values, one of 70528 and 20096). For other few rows it has fp32 sums of slices of k for 64 rows and each output; for
 * more rows, w's values, up to 2^28 of them, and x's. */
size_t sdnn_grouped_linear_workspace_bytes(int64_t n_rows, int64_t n_outputs, int64_t n_values, int32_t dtype);
sdnn_status sdnn_grouped_linear(const void *x, int64_t ldx, int32_t dtype, const uint8_t *codes, const void *scales,
                                const void *offsets, int64_t n_rows, int64_t n_outputs, int64_t n_values, int32_t group,
                                void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SDNN_H */
