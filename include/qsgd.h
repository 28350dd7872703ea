/*
 * libqsgd -- the data-parallel hot path of QSGD on one MI355X (gfx950).
 *
 * Alistarh, Grubic, Li, Tomioka, Vojnovic: "QSGD: Communication-Efficient SGD
 * via Gradient Quantization and Encoding".  The three entry points are the
 * boxed calls and the last line of Algorithm 1:
 *
 *   qsgd_encode             M <- Encode(g) = Code(Q_s(g))        (Alg. 1; Sec. 3.1)
 *   qsgd_decode_accumulate  acc <- acc + sum_l Decode(M_l)       (Alg. 1; Sec. 3.1)
 *   qsgd_sgd_step           x <- x - (eta/K) sum_l Decode(M_l)   (Alg. 1, last line)
 *
 * Plain C ABI: pointers and sizes only.  Every pointer named *_dev is device
 * memory owned by the caller; everything else is host memory.  The calls on
 * the hot path allocate no device memory: scratch comes in through
 * `workspace_dev` (the one exception is qsgd_layout_create, which uploads two
 * small tables once per layout, outside the path).  All work is queued on the HIP stream passed in (a hipStream_t cast to void*,
 * NULL = the default stream) and the calls return without waiting for it.
 *
 * Return value: 0, or a negative QSGD_ERR_* found on the host before anything
 * was queued.  Conditions only the GPU can see (message capacity exceeded, a
 * malformed message) are recorded in a status word and fetched with
 * qsgd_message_status / qsgd_workspace_status; kernels never read or write
 * outside the buffers described here, whatever the message bytes are.
 */
#ifndef QSGD_H
#define QSGD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Vector code (how the tuple (||v||, sigma, zeta) of Sec. 3.1 becomes bits). */
#define QSGD_CODE_SPARSE 0u /* Code_s : Elias(gap), sign, Elias(level) per nonzero (Sec. 3.1, App. A.2) */
#define QSGD_CODE_DENSE  1u /* Code'_s: sign, Elias(level+1) for every coordinate (App. A.3)            */
#define QSGD_CODE_FIXED  2u /* b-bit fields + sign bits, the "b-bit QSGD" of Sec. 5                     */

/* Scale of a bucket. */
#define QSGD_NORM_L2  0u    /* ||v||_2 (Eq. 2)                                    */
#define QSGD_NORM_MAX 1u    /* max_i |v_i| (Sec. 4, second variation)             */

#define QSGD_OK               0
#define QSGD_ERR_INVALID_ARG (-1) /* bad parameter, null pointer, misaligned buffer        */
#define QSGD_ERR_CAPACITY    (-2) /* message or workspace buffer too small                 */
#define QSGD_ERR_CORRUPT     (-3) /* message does not parse / header does not match params */
#define QSGD_ERR_HIP         (-4) /* a HIP runtime call failed                             */
#define QSGD_ERR_UNSUPPORTED (-5) /* valid request this build has no kernel for            */
#define QSGD_ERR_SCRATCH     (-6) /* request needs more than the built-in scratch holds    */

#define QSGD_MAX_PEERS 64u        /* largest K                                             */
#define QSGD_HEADER_BYTES 64u

/* Parameters of one Encode, and of the messages a Decode expects.
 *   n          length of the gradient vector (Sec. 2), 0 <= n < 2^32
 *   d          bucket size (Sec. 4): consecutive runs of d values are quantized
 *              independently, each with its own scale; d >= n means one bucket
 *   seed       key of the Philox-4x32-10 generator behind the rounding draws
 *   s          number of quantization levels (Sec. 3.1), 1 <= s <= 65535
 *   code, norm QSGD_CODE_*, QSGD_NORM_*
 *   stream_id  peer id and
 *   iteration  iteration number: counter words 2 and 3 of the generator, so that
 *              peers and iterations draw independently (element i uses word i%4 of
 *              the block with counter (i/4 low, i/4 high, stream_id, iteration))
 */
typedef struct qsgd_params {
  uint64_t n;
  uint64_t d;
  uint64_t seed;
  uint32_t s;
  uint32_t code;
  uint32_t norm;
  uint32_t stream_id;
  uint32_t iteration;
  uint32_t reserved; /* must be 0 */
} qsgd_params;

/* Library version (major*10000 + minor*100 + patch). Host only. */
int qsgd_version(void);

/* Text for a QSGD_ERR_* code. Host only; the string is static. */
const char *qsgd_strerror(int err);

/* Worst-case size in bytes of a message for these parameters (every coordinate
 * nonzero at the top level).  A smaller buffer may be passed to qsgd_encode when
 * the data are known to be sparse; running out is reported, never overrun.
 * Host only.  Returns 0 for invalid parameters. */
size_t qsgd_max_encoded_bytes(const qsgd_params *p);

/* Bytes of scratch the calls below need for these parameters and up to K
 * messages (K = 0 or 1 for encode-only use).  Host only; does not depend on the
 * device.  Returns 0 for invalid parameters. */
size_t qsgd_workspace_bytes(const qsgd_params *p, uint32_t K);

/* Bytes of scratch qsgd_encode needs when the message buffer has msg_capacity bytes (a
 * caller that knows its gradients to be sparse passes a buffer far below the worst case,
 * and the staging of the bucket strings can shrink with it): at most
 * qsgd_workspace_bytes(p, 1).  qsgd_encode accepts any workspace from this size up; with
 * less than the worst case, a part of the vector that codes much longer than its share of
 * msg_capacity ends the call like a message that does not fit (status QSGD_ERR_CAPACITY
 * in the header, size needed in its length field).  Host only. */
size_t qsgd_encode_workspace_bytes(const qsgd_params *p, size_t msg_capacity);

/* Encode (Alg. 1, "M^i <- Encode(g)"; Q_s: Sec. 3.1 Eq. 2 per bucket of Sec. 4;
 * Code_s / Code'_s: Sec. 3.1, App. A.2-A.3).
 *   g_dev          in : n floats, device, 16-byte aligned, finite values
 *   msg_dev        out: the message, device, 16-byte aligned, msg_capacity bytes.
 *                  Layout: 64-byte header | table of bucket word offsets
 *                  (Elias codes only) | bucket strings, each word aligned.
 *                  The used length is in the header (qsgd_message_info).
 *   workspace_dev  scratch, device, 16-byte aligned, >= qsgd_workspace_bytes(p, 1), or
 *                  >= qsgd_encode_workspace_bytes(p, msg_capacity) for sparse data;
 *                  contents on entry are ignored, calls sharing it must not overlap
 *   hip_stream     the stream the kernels are queued on
 * Errors: INVALID_ARG, CAPACITY (buffers smaller than the fixed parts), HIP,
 * UNSUPPORTED.  Payload overflow is found on the device: the header's status
 * becomes QSGD_ERR_CAPACITY and its length field says what was needed. */
int qsgd_encode(const qsgd_params *p, const float *g_dev, void *msg_dev,
                size_t msg_capacity, void *workspace_dev, size_t workspace_bytes,
                void *hip_stream);

/* qsgd_encode for callers that cannot allocate device memory and have no workspace to
 * hand over: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  The scratch is a 64 MiB array inside the library image
 * (qsgd_static_scratch_bytes()); each GPU the library runs on holds its copy until the
 * process ends.  Arguments, message and error behaviour as qsgd_encode, minus the
 * workspace; additionally QSGD_ERR_SCRATCH when qsgd_workspace_bytes(p, 1) exceeds the
 * array (nothing is queued then).  The call allocates nothing (no hipMalloc / hipFree, no
 * allocating library routine; while qsgd_timing_enable is on, timing events are taken
 * from the pool made when it was switched on).  Every call on a GPU shares that GPU's array: calls that
 * overlap in time on one GPU (different streams, different threads) race, also with
 * each other's messages; calls on one stream, or ordered by events, are safe.  Nothing
 * in the array has to survive between calls and nothing has to be cleared. */
int qsgd_encode_static(const qsgd_params *p, const float *g_dev, void *msg_dev,
                       size_t msg_capacity, void *hip_stream);
size_t qsgd_static_scratch_bytes(void);

/* Decode K messages and add them up (Alg. 1, "g^l <- Decode(M^l)" and the sum of
 * its last line):  acc_i <- acc_i + (((0 + g^0_i) + g^1_i) + ... + g^{K-1}_i),
 * g^l_i = ||v||_bucket * sgn_i * level_i / s  (Eq. 2), all in fp32.
 *   msgs_dev       host array of K device pointers (16-byte aligned messages made
 *                  with the same n, d, s, code, norm as *p), 1 <= K <= QSGD_MAX_PEERS
 *   msg_bytes      host array of K sizes: readable bytes behind each pointer (the
 *                  kernels never read past them, whatever a header claims)
 *                  Pass a message's own length where it is known: it tells how long
 *                  the strings are, which picks the decoder (the results are the same)
 *   acc_dev        in/out: n floats, device, 16-byte aligned
 *   workspace_dev  >= qsgd_workspace_bytes(p, K); word 0 receives the status
 * Errors: INVALID_ARG, CAPACITY, HIP, UNSUPPORTED on the host; a header that does
 * not match *p or a string that does not parse sets the workspace status to
 * QSGD_ERR_CORRUPT (values written for that bucket are then unspecified, nothing
 * outside acc_dev[0..n) is touched). */
int qsgd_decode_accumulate(const qsgd_params *p, const void *const *msgs_dev,
                           const size_t *msg_bytes, uint32_t K, float *acc_dev,
                           void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* The fused receive side of Alg. 1:  x_i <- fma(-(eta/K), sum_l g^l_i, x_i) with the
 * sum taken as in qsgd_decode_accumulate.  Arguments as there; x_dev in/out. */
int qsgd_sgd_step(const qsgd_params *p, const void *const *msgs_dev,
                  const size_t *msg_bytes, uint32_t K, float eta, float *x_dev,
                  void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* ---- Tensor-aware messages (Sec. 5, "Protocol": matrices with fewer than 10K
 * elements are sent unquantized, and quantization buckets are laid out per matrix).
 *
 * The gradient (and x) is an ARENA of p->n floats on the device in which tensor j
 * occupies [offsets[j], offsets[j] + sizes[j]); tensors ascend, do not overlap, and
 * start at multiples of 4 elements (16 bytes), as tensors packed with allocator
 * alignment do.  A tensor with sizes[j] < bypass_below travels as raw fp32 behind
 * the bucket strings; every other tensor is cut into buckets of d values that
 * restart at its first value (its last bucket is shorter), so no bucket mixes two
 * tensors' scales.  Draws are indexed by arena position.  Messages carry header
 * version 2; decoding needs the same layout.  d must be a multiple of 4, <= 8192.
 *
 * qsgd_layout_create builds the layout from HOST arrays and uploads two small tables
 * to the current device (it allocates device memory; the layout is immutable and may
 * be shared by any number of calls on that device); qsgd_layout_destroy frees it.
 * The other calls mirror their flat namesakes: same arguments plus the layout, same
 * ownership, same error behaviour; p->d must equal the layout's d and p->n must
 * cover its extent.  Positions of the arena outside every tensor are never read or
 * written.  Returns QSGD_ERR_UNSUPPORTED for bucket sizes the layout path does not
 * take. */
typedef struct qsgd_layout qsgd_layout;
int qsgd_layout_create(const uint64_t *offsets, const uint64_t *sizes, uint32_t T, uint64_t d,
                       uint64_t bypass_below, qsgd_layout **out);
void qsgd_layout_destroy(qsgd_layout *layout);
int qsgd_layout_info(const qsgd_layout *layout, uint64_t *buckets, uint64_t *raw_values,
                     uint64_t *extent);
size_t qsgd_layout_max_encoded_bytes(const qsgd_params *p, const qsgd_layout *layout);
size_t qsgd_layout_workspace_bytes(const qsgd_params *p, const qsgd_layout *layout, uint32_t K);
int qsgd_encode_layout(const qsgd_params *p, const qsgd_layout *layout, const float *g_dev,
                       void *msg_dev, size_t msg_capacity, void *workspace_dev,
                       size_t workspace_bytes, void *hip_stream);
int qsgd_decode_accumulate_layout(const qsgd_params *p, const qsgd_layout *layout,
                                  const void *const *msgs_dev, const size_t *msg_bytes,
                                  uint32_t K, float *acc_dev, void *workspace_dev,
                                  size_t workspace_bytes, void *hip_stream);
int qsgd_sgd_step_layout(const qsgd_params *p, const qsgd_layout *layout,
                         const void *const *msgs_dev, const size_t *msg_bytes, uint32_t K,
                         float eta, float *x_dev, void *workspace_dev, size_t workspace_bytes,
                         void *hip_stream);

/* Encode of a SLICE of a longer vector: as qsgd_encode on the p->n values at g_dev,
 * with the rounding draws of positions index_base .. index_base + p->n - 1 of the
 * whole vector (index_base a multiple of 4, else QSGD_ERR_INVALID_ARG; any code and any
 * bucket size qsgd_encode takes).  If index_base is a multiple of the bucket size, the
 * buckets and levels are exactly those the whole vector would get. */
int qsgd_encode_slice(const qsgd_params *p, uint64_t index_base, const float *g_dev,
                      void *msg_dev, size_t msg_capacity, void *workspace_dev,
                      size_t workspace_bytes, void *hip_stream);

/* ---- Double-buffered pass (Sec. 5, "Protocol": quantization and communication are
 * double buffered so that they overlap with computation).  The vector of p->n values is
 * cut into chunks of chunk_elems (a multiple of the bucket size and of 4; any code and
 * bucket size the flat calls take).  For every chunk the K
 * peers' slices g_dev[k] + offset are encoded (peer k with stream_id p->stream_id + k)
 * on one internal stream, then decoded, summed and applied to x_dev + offset on a second
 * one, while the next chunk is already being encoded; msg_dev holds 2*K device buffers
 * of msg_capacity bytes each (two sets used alternately; size them with
 * qsgd_max_encoded_bytes for n = chunk_elems), and the two workspaces (distinct, each
 * workspace_bytes >= qsgd_workspace_bytes for n = chunk_elems) serve the encode and the
 * decode side.  The work starts after what is queued on hip_stream at the time of the
 * call, and hip_stream continues after the last chunk.  x ends up exactly as after one
 * qsgd_sgd_step over the K whole-vector messages.  Errors as the calls it is made of:
 * sizes and parameters of every chunk are checked before anything is queued, so a
 * negative return leaves x untouched (only a failing HIP call can end the pass half way;
 * the internal streams may then still hold work: synchronise the device).
 * qsgd_pipeline_create makes the two streams (default priority) and five events on the
 * current device; calls on one pipeline object must not overlap. */
typedef struct qsgd_pipeline qsgd_pipeline;
int qsgd_pipeline_create(qsgd_pipeline **out);
void qsgd_pipeline_destroy(qsgd_pipeline *pl);
int qsgd_pipeline_step(qsgd_pipeline *pl, const qsgd_params *p, uint64_t chunk_elems,
                       const float *const *g_dev, uint32_t K, float eta, float *x_dev,
                       void *const *msg_dev, size_t msg_capacity, void *enc_workspace_dev,
                       void *dec_workspace_dev, size_t workspace_bytes, void *hip_stream);

/* ---- A layer in 8 bits: what makes the gradient that qsgd_encode takes.  The quantizer of
 * Sec. 3.1 with s = 127 levels and the largest magnitude as scale (Sec. 4), a bucket being a
 * row or a column of a matrix; the product of two such matrices in integers; a linear layer
 * made of them with its gradients; and dropout from the same counter-based generator.
 * All draws are reproducible from their key and position, no mask or generator state is stored.
 *
 * The calls queue kernels on hip_stream on the current device, whose memory the arguments are in, allocate
 * nothing and may be captured.  An output or a workspace must not overlap another argument, except where said;
 * outputs that do are refused with QSGD_ERR_INVALID_ARG (column ranges of one larger matrix do not
 * overlap).  QSGD_ERR_UNSUPPORTED: more work than a launch can count (2^32 blocks of eight columns of dropout,
 * 2^24 rows of more than 2048 columns of the quantizer and 2^26 of any, 2^30 columns quantized by columns, 2^26 rows of
 * an operand, rows of levels 2^23 bytes apart, 2^38 results of a product).
 *
 * The *_workspace_bytes below are host only and, among sizes that a call takes, never shrink when one grows: a
 * workspace made for the largest batch, or for the largest of several layers in each of the three sizes, serves the smaller
 * ones.  What one call itself needs can be less, and a workspace is refused only below that.
 */

/* Element types of a matrix. */
#define QSGD_TYPE_F32  0u
#define QSGD_TYPE_BF16 1u
#define QSGD_TYPE_F16  2u
#define QSGD_TYPE_I8   3u

#define QSGD_ROUND_NEAREST    0u /* to the nearest level, ties to the even one              */
#define QSGD_ROUND_STOCHASTIC 1u /* to one of the two levels around the value, unbiased      */

/* A matrix in device memory: element (r, c) is at data_dev[r * ld + c].  rows, cols < 2^31,
 * rows * ld < 2^46.  ld >= cols; the data are aligned to their element's size.  Matrices of QSGD_TYPE_I8
 * are aligned to 16 bytes, ld is a multiple of 16, and the bytes of a row up to the next
 * multiple of 16 are readable; what stands there changes no result and is not written.
 * data_dev may be NULL where rows or cols is 0. */
typedef struct qsgd_matrix {
  void *data_dev;
  uint64_t rows, cols, ld;
  uint32_t type;
  uint32_t reserved; /* must be 0 */
} qsgd_matrix;

/* The draws of a matrix: element (r, c) has the half-word c % 8 (two to a word, the low one
 * first) of the Philox-4x32-10 block with counter (c / 8, row_base + r, stream_id, iteration)
 * and key seed.  A slice of rows passes the number of its first row as row_base
 * (row_base + rows <= 2^32).  iteration_dev, a word in device memory or NULL, is added to
 * iteration when the kernels run, so that a captured graph draws anew at each replay; it must
 * not lie in an output (refused with QSGD_ERR_INVALID_ARG).
 *
 * A draw is named by (seed, stream_id, iteration), row and column, and by nothing else: calls with
 * the same name draw the same half-words, whatever for.  That is what makes qsgd_dropout_backward
 * find the mask of qsgd_dropout; any two others that are to be independent must differ in one of
 * the three.  qsgd_linear_backward takes stream_id, stream_id + 1 and stream_id + 2 (modulo 2^32),
 * the other calls stream_id alone, and the blocks of qsgd_encode (stream_id: the peer) are those
 * of row 0.  With one name for dropout and for the quantizer of what it leaves, for instance, the
 * kept elements are those of large draws, which round up too rarely: levels are p / 2 too near to
 * zero in the mean, and the gradient is biased.
 * A way that uses no draw twice: a seed for the codec; one for each dropout, with stream_id = peer;
 * one for each layer, with stream_id = 4 peer for qsgd_linear_backward and 4 peer + 3 for its
 * stochastic qsgd_linear_forward or qsgd_quantize; and the step as iteration. */
typedef struct qsgd_draws {
  uint64_t seed;
  uint32_t stream_id;
  uint32_t iteration;
  uint32_t row_base;
  uint32_t reserved; /* must be 0 */
  const uint32_t *iteration_dev;
} qsgd_draws;

/* Dropout:  y = residual + keep * x * 65536 / (65536 - D),  D = rint(65536 p), 0 <= p <= 1;
 * keep is whether the element's draw h >= D, so an element is dropped with probability D / 65536
 * exactly and E y = residual + x (p = 1 or nearest to it drops everything).  A dropped element
 * contributes +0 whatever its value.  Computed in fp32, rounded once to y's type.  x, residual
 * (NULL: none) and y have one shape and one type of F32, BF16, F16; y may be x or residual
 * itself (same data_dev and ld), otherwise it must not overlap them. */
int qsgd_dropout(const qsgd_draws *draws, float p, const qsgd_matrix *x,
                 const qsgd_matrix *residual, const qsgd_matrix *y, void *hip_stream);

/* Its gradient with the same draws and p:  dx = keep * dy * 65536 / (65536 - D).  (The gradient
 * of the residual is dy.)  dx may be dy itself. */
int qsgd_dropout_backward(const qsgd_draws *draws, float p, const qsgd_matrix *dy,
                          const qsgd_matrix *dx, void *hip_stream);

/* Quantizer by rows, by columns, or both:  with m the largest magnitude of the row (column),
 *   scale = m / 127,  t = |x| fl(127 / m) in fp32,  level = sgn(x) rint(t)                 (nearest)
 *                                                   level = sgn(x) (floor(t) + [u < t - floor(t)])  (stochastic)
 * with u = (h + 1/2) / 65536, h the element's draw (the same one in both forms); at most 127.
 * A row with m < 2^-119 counts as zero (scale 0, levels 0); one that holds an infinity or a NaN
 * gets scale NaN and levels 0, so that whatever is computed from it is NaN.
 *   x           F32, BF16 or F16
 *   rows        out: levels, I8, the shape of x (or NULL); row_scale_dev: x->rows floats
 *   columns     out: levels TRANSPOSED, I8, x->cols rows of x->rows values (or NULL);
 *               column_scale_dev: x->cols floats
 *   workspace   device, 16-byte aligned, >= qsgd_quantize_workspace_bytes(x->rows, x->cols);
 *               not used (NULL, 0) without columns
 *   draws       may be NULL for QSGD_ROUND_NEAREST */
size_t qsgd_quantize_workspace_bytes(uint64_t rows, uint64_t cols);
int qsgd_quantize(const qsgd_draws *draws, uint32_t rounding, const qsgd_matrix *x,
                  const qsgd_matrix *rows, float *row_scale_dev, const qsgd_matrix *columns,
                  float *column_scale_dev, void *workspace_dev, size_t workspace_bytes,
                  void *hip_stream);

/* Product of 8-bit matrices:  y[m][n] = (sum_k a[m][k] b[n][k]) a_scale[m] b_scale[n] + bias[n].
 * The sum is exact (32-bit integers, joined in 64 bits where they could pass); the factors are
 * applied in fp32, a's scale first, b's and the bias in one rounding, and the result is rounded once
 * to y's type; it overflows only where its value does (a scale below 2^-126 may vanish).
 *   a  M x K, I8, with M scales;  b  N x K, I8, with N scales;  bias_dev  N floats or NULL
 *   y  M x N, F32, BF16 or F16; must not overlap the operands
 *   workspace  device, 16-byte aligned, >= qsgd_int_matmul_workspace_bytes(M, N, K), calls sharing
 *              it must not overlap; NULL where that is 0
 * QSGD_ERR_UNSUPPORTED: rows of the operands 2^23 bytes apart or more. */
size_t qsgd_int_matmul_workspace_bytes(uint64_t M, uint64_t N, uint64_t K);
int qsgd_int_matmul(const qsgd_matrix *a, const float *a_scale_dev, const qsgd_matrix *b,
                    const float *b_scale_dev, const float *bias_dev, const qsgd_matrix *y,
                    void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* Linear layer, forward:  y = Q(x) W^T + bias, Q the quantizer by rows (tokens), W the weights as
 * qsgd_quantize left them by rows (outputs x inputs, a scale per output).  x, y: one type of
 * F32, BF16, F16.  The result is that of qsgd_quantize and qsgd_int_matmul. */
size_t qsgd_linear_forward_workspace_bytes(uint64_t tokens, uint64_t outputs, uint64_t inputs);
int qsgd_linear_forward(const qsgd_draws *draws, uint32_t rounding, const qsgd_matrix *x,
                        const qsgd_matrix *w, const float *w_scale_dev, const float *bias_dev,
                        const qsgd_matrix *y, void *workspace_dev, size_t workspace_bytes,
                        void *hip_stream);

/* Its gradients, from the unquantized x (tokens x inputs), w (outputs x inputs) and dy (tokens x
 * outputs), one type of F32, BF16, F16:
 *   dx = Q_row(dy) Q_col(w)      that type         (or NULL)
 *   dw = Q_col(dy)^T Q_col(x)    F32: the gradient that qsgd_encode takes   (or NULL)
 *   db = sum over the tokens of dy, in fp32        (or NULL)
 * dy draws with stream_id, w with stream_id + 1 (its rows counted from 0), x with
 * stream_id + 2.  With stochastic rounding the factors are independent, so that E dx = dy w and
 * E dw = dy^T x: unbiased estimates of the gradient, as Algorithm 1 asks of g, where x, w and dy
 * do not depend on the same draws themselves (see qsgd_draws). */
size_t qsgd_linear_backward_workspace_bytes(uint64_t tokens, uint64_t outputs, uint64_t inputs);
int qsgd_linear_backward(const qsgd_draws *draws, uint32_t rounding, const qsgd_matrix *x,
                         const qsgd_matrix *w, const qsgd_matrix *dy, const qsgd_matrix *dx,
                         const qsgd_matrix *dw, float *db_dev, void *workspace_dev,
                         size_t workspace_bytes, void *hip_stream);

/* Reads a message header from a HOST copy of (at least) its first 64 bytes.
 * Fills *out (seed is not stored: 0) and *total_bytes (either may be NULL).
 * Returns 0, QSGD_ERR_CORRUPT (not a header), or the status the encoder left
 * (QSGD_ERR_CAPACITY: *total_bytes is the size that would have been needed). */
int qsgd_message_info(const void *header_host, qsgd_params *out, uint64_t *total_bytes);

/* Convenience: waits for `hip_stream`, copies the header of msg_dev to the host
 * and returns what qsgd_message_info returns (or QSGD_ERR_HIP). */
int qsgd_message_status(const void *msg_dev, uint64_t *total_bytes, void *hip_stream);

/* Waits for `hip_stream` and returns the status word the last decode call left
 * in workspace_dev (0 or QSGD_ERR_CORRUPT), or QSGD_ERR_HIP. */
int qsgd_workspace_status(const void *workspace_dev, void *hip_stream);

/* Kernel timing for benchmarks: while enabled, every kernel launch of the
 * library is bracketed by HIP events on its own stream.  qsgd_timing_get waits
 * for the recorded events and reports, for kernels whose name starts with
 * `prefix`, the summed duration in milliseconds and the launch count since the
 * last reset.  Off by default; not for use inside stream capture. */
int qsgd_timing_enable(int on);
int qsgd_timing_reset(void);
int qsgd_timing_get(const char *prefix, double *total_ms, uint64_t *launches);

/* Measurement aid, not part of the method: a plain copy kernel (16-byte loads and
 * stores, grid-stride) of `bytes` bytes (a multiple of 16) from src_dev to dst_dev,
 * both device pointers aligned to 16 bytes, on `hip_stream` (streaming accesses, one
 * contiguous 16 KiB piece per workgroup).  It gives the copy ceiling of the machine the
 * codec is compared with, and a kernel of known HBM traffic that hardware counters can
 * be calibrated against.  Timed as "copy_probe".
 * Returns 0, QSGD_ERR_INVALID_ARG or QSGD_ERR_HIP. */
int qsgd_copy_probe(void *dst_dev, const void *src_dev, size_t bytes, void *hip_stream);

/* Measurement aid, not part of the method: the same copy with ONE 4-byte load and one
 * 4-byte store per lane (bytes a multiple of 4), the request size of the kernels that read
 * message strings word by word.  A second kernel of known traffic, so that the factors of
 * the hardware counters are known for both request sizes.  Timed as "copywords_probe". */
int qsgd_copy_probe_words(void *dst_dev, const void *src_dev, size_t bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* QSGD_H */
