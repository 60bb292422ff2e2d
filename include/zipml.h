/*
 * libzipml -- double-sampled low-precision minibatch SGD for least squares on AMD MI355X (gfx950).
 *
 * The method is that of "ZipML: Training Models with End-to-End Low Precision"
 * (arXiv 1611.05402): every sample row is stochastically quantised twice, independently, to
 * b-bit per-feature levels (Sec. 2.1, Supp. A.3), and each minibatch step uses the unbiased
 * double-sampled gradient  g = mean_i Q1(a_i) (Q2(a_i)^T x - b_i)  (Sec. 2.2, eq. (5)), optionally
 * with the model and the gradient stochastically quantised as well (Supp. C-E).
 *
 * General conventions
 *   - Plain C ABI.  Pointers named *_dev are DEVICE pointers owned by the caller; the library never
 *     allocates or frees device memory and keeps no pointer of the caller's after a call returns
 *     (zipml_loss keeps some pinned host memory of its own, see there).  Pointers named
 *     *_host are host pointers.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All device work is
 *     enqueued on it.  Calls that return a host value (zipml_loss, zipml_sgd_status, zipml_scan_status,
 *     the OPTIMAL mode of zipml_levels) synchronise that stream; every other call is asynchronous.
 *   - Every call returns ZIPML_OK (0) or a negative error code; nothing aborts or throws across the
 *     boundary.  Argument errors are detected before any work is enqueued.
 *   - A is row-major fp32 with leading dimension lda >= d.  Level tables are [d][2^bits] fp32,
 *     non-decreasing along the second axis.  All device pointers must be 16-byte aligned.
 *   - The packed layout of the quantised copies is private to the library (copy 1 is stored
 *     feature-major for the gradient pass, copy 2 sample-major for the dot-product pass, both in
 *     units of 32 codes); zipml_unpack_codes is its only definition.
 *   - Random numbers: Philox4x32-10, key = seed, counter = (row, feature / 4, epoch * 256 + stream),
 *     output word feature % 4, the top 24 bits as a uniform in [0,1).  Streams 1, 2 are the two
 *     sample quantisations (row = sample index), 3 and 4 the model and gradient quantisations
 *     (row = step index within the epoch), 16 and up the stored activations and the rows of codes.  epoch must be < 2^24.
 */
#ifndef ZIPML_H
#define ZIPML_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------------------------- */
#define ZIPML_OK            0
#define ZIPML_EINVAL       -1   /* bad argument value (sizes, bits, batch, NULL pointer)          */
#define ZIPML_EALIGN       -2   /* a device pointer is not 16-byte aligned                        */
#define ZIPML_ERANGE       -3   /* integer dot product could overflow int32 for these sizes       */
#define ZIPML_EWORKSPACE   -4   /* workspace missing or smaller than zipml_workspace_bytes()      */
#define ZIPML_ELAUNCH      -5   /* the HIP runtime refused a launch or copy                       */
#define ZIPML_EUNSUPPORTED -6   /* valid request that this build does not implement               */
#define ZIPML_ETIMEOUT     -7   /* a wait inside an epoch kernel or a recurrence gave up          */

/* ---- modes and flags ---------------------------------------------------------------------- */
#define ZIPML_UNIFORM 0          /* 2^bits evenly spaced levels on [lo_j, hi_j]    (Sec. 2.1)     */
#define ZIPML_OPTIMAL 1          /* variance-optimal levels by dynamic programming (Sec. 3)       */
#define ZIPML_GREEDY 2           /* the same over the candidates a greedy search leaves (Sec. 3.2) */

#define ZIPML_RANGE_GIVEN 1      /* zipml_levels: lo_dev / hi_dev are inputs                      */
#define ZIPML_SYMMETRIC   2      /* zipml_levels: range [-M_j, M_j], M_j = max(|min|, |max|)
                                    (Supp. A.3 "Column Scaling")                                  */

#define ZIPML_SGD_STEPWISE 1     /* zipml_sgd_epoch: two launches per step instead of one
                                    persistent launch per epoch (same arithmetic)                 */
#define ZIPML_SGD_AVERAGED 2     /* zipml_sgd_epoch: the averaged estimator
                                    1/2 [Q1 (Q2^T x - b) + Q2 (Q1^T x - b)]  (Supp. B.2, footnote) */
#define ZIPML_SGD_PRODUCTION 4   /* zipml_debug_step: run the step in the launch and step loop that
                                    zipml_sgd_epoch takes for this shape (see zipml_debug_step)     */

const char *zipml_strerror(int code);

/* Bytes of ONE packed copy of an n x d matrix at `bits` bits per value, padding included
 * (n is rounded up to a multiple of 64, d to a multiple of 32).  0 if the arguments are invalid. */
size_t zipml_packed_bytes(int64_t n, int64_t d, int bits);

/* Bytes of device workspace that zipml_levels, zipml_sgd_epoch, zipml_debug_step and zipml_loss
 * need for a problem of this shape (one buffer serves all of them, one call at a time).
 * n_candidates may be 0 if neither ZIPML_OPTIMAL nor ZIPML_GREEDY is used (with it, the size
 * includes the bin moments, 24 d n_candidates bytes, and 64 MiB for partial copies of them). */
size_t zipml_workspace_bytes(int64_t n, int64_t d, int bits, int64_t batch, int n_candidates);

/* Per-feature quantisation levels.
 *   Sec. 2.1 (levels partition the scaled range), Supp. A.3 "Column Scaling" (one range per
 *   feature from the column min/max), Sec. 3.1-3.2 (variance-optimal levels: one scan of the data
 *   into n_candidates equal bins per feature, then the dynamic program T(k,m) on the bin edges).
 * Unless ZIPML_RANGE_GIVEN, lo_dev[d] / hi_dev[d] are written with the column ranges.
 * levels_dev[d][2^bits] is written.  grid_idx_dev[d][2^bits] (optional, may be NULL) receives the
 * integer grid position of every level: c for UNIFORM, the chosen bin edge for OPTIMAL, so that
 * level = lo_j + (hi_j - lo_j) * grid_idx / grid_max with grid_max = 2^bits - 1 or n_candidates.
 * mean_variance_host (optional, OPTIMAL and GREEDY only) receives the objective of eq. (6)
 * averaged over features.  UNIFORM is asynchronous.  OPTIMAL runs the dynamic program on the device
 * when its tables fit in on-chip memory (then only a request for mean_variance_host synchronises
 * the stream); otherwise it copies the bin moments to the host, runs the dynamic program on the
 * host cores and copies the levels back, which synchronises the stream.
 * GREEDY (Sec. 3.2, "2-Approximation in Almost-Linear Time"; supplement, Algorithm 1 with
 * gamma = 1, delta = 1): the bins are first merged greedily into at most 4 (2^bits - 1) + 1
 * intervals per feature, whose end points are the only candidates of the dynamic program; the
 * levels are within the factor the paper gives of OPTIMAL's, for a dynamic program over ~4 * 2^bits
 * instead of n_candidates points.  With n_candidates <= 4 (2^bits - 1) + 1 it is OPTIMAL.  Device
 * only: ZIPML_EUNSUPPORTED if the tables do not fit (8 bits with more than 1021 candidates).
 * bits in 1..8; OPTIMAL and GREEDY need 2^bits - 1 <= n_candidates <= 4096. */
int zipml_levels(void *stream, const float *A_dev, int64_t n, int64_t d, int64_t lda, int bits,
                 int mode, int flags, int n_candidates, float *lo_dev, float *hi_dev,
                 float *levels_dev, uint16_t *grid_idx_dev, double *mean_variance_host,
                 void *workspace_dev, size_t workspace_bytes);

/* Two independent stochastic quantisations of rows [row0, row0 + n_rows) of an n_total x d matrix
 * (Sec. 2.1: value v between neighbouring levels l <= v <= u goes to u with probability
 * (v - l)/(u - l), evaluated in fp32; Sec. 2.2: two independent copies).  A_dev points at the
 * first of the n_rows rows.  Values outside the level range are clamped to it.  packed1_dev and
 * packed2_dev each hold zipml_packed_bytes(n_total, d, bits) bytes; calls for disjoint row ranges
 * fill disjoint parts, so a large matrix can be quantised chunk by chunk.  row0 must be a multiple
 * of 32, and so must n_rows unless the chunk ends at n_total. */
int zipml_quantize(void *stream, const float *A_dev, int64_t n_rows, int64_t d, int64_t lda,
                   int64_t row0, int64_t n_total, const float *levels_dev, int bits, uint64_t seed,
                   uint32_t epoch, void *packed1_dev, void *packed2_dev);

/* The same two copies in the other layout each, for the symmetrised estimator: packed1s_dev gets
 * copy 2 in the layout of packed1, packed2s_dev copy 1 in the layout of packed2.  The draws are
 * those of zipml_quantize with the same (seed, epoch): zipml_unpack_codes(packed1s, copy = 1)
 * returns the codes of copy 2, and (packed2s, copy = 2) those of copy 1. */
int zipml_quantize_swapped(void *stream, const float *A_dev, int64_t n_rows, int64_t d, int64_t lda,
                           int64_t row0, int64_t n_total, const float *levels_dev, int bits,
                           uint64_t seed, uint32_t epoch, void *packed1s_dev, void *packed2s_dev);

/* Compact storage of the two samples (Sec. 2.2, "Overhead of Storing Samples"): the two
 * quantisations of a value differ by at most one level, so a base level and one bit per sample
 * hold both, bits + 2 bits per value instead of 2 * bits.  packed_a_dev and packed_b_dev are the
 * two copies in the SAME layout -- (packed2s, packed2): copy 1 and copy 2 sample-major, or
 * (packed1, packed1s): copy 1 and copy 2 feature-major, see zipml_quantize_swapped -- and
 * compact_dev holds zipml_compact_bytes(n, d, bits) bytes in two planes: first the smaller of the
 * two codes of every value, a packed array in the layout of the copies (bits / (bits + 2) of the
 * record); then, per unit of 32 values in the same order, a pair of dwords of bits saying which
 * values of copy a / copy b sit one level above it.  A storage and transfer format, restored bit
 * for bit by zipml_compact_decode; zipml_sgd_epoch_compact runs on the sample-major record as it is.  zipml_compact_encode synchronises the stream and
 * returns ZIPML_EINVAL if some pair of codes differs by more than one level (the arrays are then
 * not two samples of the same values); it uses 256 bytes of workspace. */
size_t zipml_compact_bytes(int64_t n, int64_t d, int bits);
int zipml_compact_encode(void *stream, const void *packed_a_dev, const void *packed_b_dev, int64_t n,
                         int64_t d, int bits, void *compact_dev, void *workspace_dev,
                         size_t workspace_bytes);
int zipml_compact_decode(void *stream, const void *compact_dev, int64_t n, int64_t d, int bits,
                         void *packed_a_dev, void *packed_b_dev);

/* zipml_sgd_epoch for very large minibatches reading the COMPACT record alone (Sec. 2.2, "Overhead
 * of Storing Samples"): compact_dev is what zipml_compact_encode writes for the two copies in the
 * sample-major layout, (packed2s, packed2) -- copy 1 from zipml_quantize_swapped, copy 2 from
 * zipml_quantize.  A step then reads bits + 2 instead of 2 * bits bits per value; the gradient pass
 * turns its operand on the chip.  Same estimator and arithmetic as zipml_sgd_epoch on the packed
 * copies (the model after the epoch is bit-identical).  Built for bits = 8, evenly spaced levels,
 * the fp32 model, minibatches of at least 16384 samples (a multiple of 64) and 513 to 2048
 * features; ZIPML_EUNSUPPORTED otherwise (for level tables that turn out not to be evenly spaced:
 * through zipml_sgd_status).  Asynchronous; workspace as for zipml_sgd_epoch. */
int zipml_sgd_epoch_compact(void *stream, const void *compact_dev, const float *levels_dev,
                            const float *b_dev, int64_t n, int64_t d, int bits, float *x_dev,
                            int64_t batch, float lr, void *workspace_dev, size_t workspace_bytes);

/* One epoch of double-sampled minibatch SGD on F(x) = 1/(2n) sum_i (a_i^T x - b_i)^2
 * (Sec. 2 and eq. (5); the minibatch gradient is the mean over `batch` consecutive samples; the
 * n / batch steps run in storage order).  x_dev[d] is the fp32 master model, updated in place:
 * x <- x - lr * g every step (Supp. E: the update is in full precision).
 *   model_bits = grad_bits = 0: full-precision (fp32) model, residuals and gradient.  The sums
 *     over features and over samples are accumulated as integers (fixed-point partial sums, and
 *     for evenly spaced levels exact integer sums of codes times fixed-point digits) or added in a
 *     fixed order, so the result does not depend on the order in which workgroups finish: two calls
 *     with the same arguments give the same bits.  The digits keep every fp32 bit of residuals, model
 *     and levels down to 2^-35 of the largest residual and 2^-22 of a bound on the largest product of
 *     model and spacing; at 2, 4 and 8 bits, minibatches a multiple of 64 and more than 256 features
 *     they end 29 bits below these.  A problem that one workgroup holds (up to 256 features) runs in
 *     fp32, or on digits of the first kind, to 2^-35 of the largest throughout.
 *   model_bits in 2..8: the model is stochastically quantised each step with row scaling
 *     (Supp. A.3 eq. (quant2), Supp. C), s = 2^(model_bits-1) - 1 magnitude intervals, and the dot
 *     product becomes an exact integer sum of grid_idx * model code; this needs grid_idx_dev and a
 *     level grid shared by all features: level value = grid_lo + grid_step * grid_idx.
 *   grad_bits in 2..8 (needs model_bits > 0): the mean gradient is quantised the same way before
 *     the update (Supp. D, E).
 * grid_max is the largest grid index (2^bits - 1 for UNIFORM levels, n_candidates for OPTIMAL);
 * ZIPML_ERANGE if grid_max * s * d could exceed int32.
 * batch must divide n and be 4, 8, 16 or a multiple of 32.  A minibatch of up to 2048 / GQ samples
 * (GQ = 1, 2 or 4 groups of 32 features per workgroup; 1024 samples at d = 2048) is one exchange
 * between the workgroups; larger ones -- up to the whole data set, i.e. gradient descent with
 * double sampling -- are supported for the fp32 model with evenly spaced 2-, 4- or 8-bit levels
 * and batch a multiple of 64 (taken in chunks by replicas of the workgroups, or by workgroups that
 * own samples instead of features); otherwise ZIPML_EUNSUPPORTED, which for level tables that
 * turn out not to be evenly spaced arrives through zipml_sgd_status with x_dev left untouched.
 * The call is asynchronous; a failed grid-wide wait is reported by zipml_sgd_status (ZIPML_ETIMEOUT):
 * the kernel then still runs to its end, and x_dev holds undefined values afterwards.
 * The workgroups of an epoch kernel wait for each other, so they must all be resident at once: the
 * library sizes the grid for that and refuses the launch (ZIPML_ELAUNCH) if the device cannot hold
 * it, but kernels of other streams that occupy the compute units at the same time can still keep
 * workgroups out -- two epoch calls on different streams of one device must not overlap; if they do,
 * the waits give up (ZIPML_ETIMEOUT) rather than hang. */
int zipml_sgd_epoch(void *stream, const void *packed1_dev, const void *packed2_dev,
                    const float *levels_dev, const uint16_t *grid_idx_dev, float grid_lo,
                    float grid_step, int grid_max, const float *b_dev, int64_t n, int64_t d,
                    int bits, float *x_dev, int64_t batch, float lr, int grad_bits, int model_bits,
                    uint64_t seed, uint32_t epoch, int flags, void *workspace_dev,
                    size_t workspace_bytes);

/* The same epoch for the least-squares SVM objective
 *   1/(2n) sum_i (a_i^T x - b_i)^2 + (c/2) ||x||^2,  b_i in {-1, +1}
 * ("Extension to Classification Models", Least Squares Support Vector Machines): the gradient of a
 * step gets the additional term c * x, taken in full precision:  x <- x - lr * (g + l2 * x).
 * Full-precision (fp32) model only; l2 >= 0; everything else as in zipml_sgd_epoch. */
int zipml_sgd_epoch_l2(void *stream, const void *packed1_dev, const void *packed2_dev,
                       const float *levels_dev, const float *b_dev, int64_t n, int64_t d, int bits,
                       float *x_dev, int64_t batch, float lr, float l2, int flags,
                       void *workspace_dev, size_t workspace_bytes);

/* The same epoch with the proximal step of the general update of Sec. 2,
 *   x <- prox_{lr R}( x - lr * (g + l2 * x) ),  prox_{lr R}(v) = argmin_u 1/2 ||u - v||^2 + lr R(u),
 * for the regularisers that act coordinate by coordinate:
 *   ZIPML_PROX_L1    R(x) = prox_coef * ||x||_1          (soft threshold at lr * prox_coef)
 *   ZIPML_PROX_L2SQ  R(x) = prox_coef / 2 * ||x||_2^2    (v / (1 + lr * prox_coef))
 *   ZIPML_PROX_BOX   the constraint ||x||_inf <= prox_coef (clamp)
 *   ZIPML_PROX_NONE  R = 0 (then the call is zipml_sgd_epoch_l2).
 * Full-precision (fp32) model only; prox_coef >= 0; everything else as in zipml_sgd_epoch_l2.
 * (Regularisers that need a norm of the whole model -- the unsquared l2 norm, an l2 ball -- are
 * not provided.) */
#define ZIPML_PROX_NONE 0
#define ZIPML_PROX_L1   1
#define ZIPML_PROX_L2SQ 2
#define ZIPML_PROX_BOX  3
int zipml_sgd_epoch_prox(void *stream, const void *packed1_dev, const void *packed2_dev,
                         const float *levels_dev, const float *b_dev, int64_t n, int64_t d, int bits,
                         float *x_dev, int64_t batch, float lr, float l2, int prox, float prox_coef,
                         int flags, void *workspace_dev, size_t workspace_bytes);

/* The same epoch with the symmetrised estimator (Supp. B.2 "Double Sampling", footnote: lower variance at no extra
 * randomness; the form the authors report running):
 *   g = 1/2 mean_i [ Q1(a_i) (Q2(a_i)^T x - b_i) + Q2(a_i) (Q1(a_i)^T x - b_i) ],
 * which needs both copies in both layouts: packed1s_dev / packed2s_dev from
 * zipml_quantize_swapped.  fp32 model; 2-, 4- or 8-bit evenly spaced levels; batch a multiple
 * of 64; more than 256 features (otherwise ZIPML_EUNSUPPORTED, through the status word if it is
 * the level tables that do not qualify).  l2 as in zipml_sgd_epoch_l2 (0 for plain least squares).
 * Large minibatches are taken as in zipml_sgd_epoch (chunks, replicas, sample owners). */
int zipml_sgd_epoch_avg(void *stream, const void *packed1_dev, const void *packed2_dev,
                        const void *packed1s_dev, const void *packed2s_dev, const float *levels_dev,
                        const float *b_dev, int64_t n, int64_t d, int bits, float *x_dev,
                        int64_t batch, float lr, float l2, int flags, void *workspace_dev,
                        size_t workspace_bytes);

/* For callers that cannot allocate device memory -- code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc: zipml_sgd_epoch with its workspace taken from a fixed
 * array of ZIPML_STATIC_WORKSPACE_BYTES bytes that is part of the library's code object (every GPU
 * the library runs on holds its own copy until the process ends).  The call allocates and frees
 * nothing and calls no allocating routine; the address of the array on the current device is
 * looked up on the first call on that device (make that call outside a capture).
 * Arguments as zipml_sgd_epoch, without the workspace.  status_dev (device, one int, 4-byte
 * aligned, required) receives what zipml_sgd_status would return for the call -- ZIPML_OK,
 * ZIPML_ETIMEOUT or ZIPML_EUNSUPPORTED -- once the work enqueued on the stream is done.
 * ZIPML_EWORKSPACE (with a line on stderr that names both sizes) if
 * zipml_workspace_bytes(n, d, bits, batch, 0) exceeds ZIPML_STATIC_WORKSPACE_BYTES.
 * All calls on one GPU share the one array, and it keeps what the last call left in it (a call
 * clears what it needs cleared): calls that overlap in time on one GPU -- two streams, two host
 * threads -- race and give undefined results; serialise them or use zipml_sgd_epoch. */
#define ZIPML_STATIC_WORKSPACE_BYTES (8u << 20)
int zipml_sgd_epoch_static(void *stream, const void *packed1_dev, const void *packed2_dev,
                           const float *levels_dev, const uint16_t *grid_idx_dev, float grid_lo,
                           float grid_step, int grid_max, const float *b_dev, int64_t n, int64_t d,
                           int bits, float *x_dev, int64_t batch, float lr, int grad_bits,
                           int model_bits, uint64_t seed, uint32_t epoch, int flags, int *status_dev);

/* Waits for the stream and returns the status word the last zipml_sgd_epoch / zipml_debug_step
 * left in this workspace: ZIPML_OK or ZIPML_ETIMEOUT. */
int zipml_sgd_status(void *stream, const void *workspace_dev, size_t workspace_bytes);

/* Loss F(x) = 1/(2n) sum_i (a_i^T x - b_i)^2 (Sec. 1 eq. (1) with the square loss).  With A_dev
 * the exact fp32 rows are used; with A_dev == NULL the rows are decoded from one packed copy
 * (`copy` = 1 or 2) and levels_dev.  Dot products in fp32 or better (levels and model keep at least
 * their fp32 bits: products and sums in fp32, or in exact integer sums for evenly spaced levels),
 * squares and their sum in fp64.  Synchronises the stream and writes *loss_host; ZIPML_ELAUNCH, with
 * nothing enqueued, on a stream that is being captured.  The partial sums arrive in pinned host memory of
 * 16 KiB a call in flight, of which the library keeps up to eight for later calls until the process
 * ends (its one allocation; nothing of it is on the device). */
int zipml_loss(void *stream, const float *A_dev, int64_t lda, const void *packed_dev, int copy,
               const float *levels_dev, int bits, const float *b_dev, const float *x_dev,
               int64_t n, int64_t d, double *loss_host, void *workspace_dev,
               size_t workspace_bytes);

/* ---- layers whose activations are stored in 8 bits ------------------------------------------
 * What a layer keeps of its forward pass for its backward pass, in 8 bits by the stochastic rounding of Sec. 2.1, and the
 * two backward passes that read it: a linear layer's weight gradient and a gated linear recurrence's.  All calls are
 * asynchronous and may be captured in a graph.  A workspace needs no preparation and keeps nothing from call to call; it may
 * be shared by all calls that follow one another on a stream, not by calls that overlap.  */

#define ZIPML_F32  0             /* element types of activations and gradients                     */
#define ZIPML_BF16 1

/* Bytes of a rows x cols tensor stored in 8 bits (33/32 of a byte a value, cols rounded up to a
 * multiple of 32); 0 if the arguments are invalid.  Layout (public): codes, int8 [rows][padded], then one
 * byte for each 32 columns of a row, [rows][padded / 32], the exponent e of the group's step 2^e plus 127.
 * value = code * 2^e, which bf16 and fp32 hold exactly. */
size_t zipml_act_bytes(int64_t rows, int64_t cols);

/* Stores rows x cols values in 8 bits by stochastic rounding (Sec. 2.1's quantiser on evenly spaced
 * levels, per 32 columns of a row): e is the least integer >= -126 with max |v| <= 127 * 2^e, code =
 * floor(v * 2^-e + (k + 1/2) / 2^16), evaluated in fp32, k a 16-bit draw, so a decoded value is v in
 * expectation (to 2^-17 of a step).  A group that holds an infinity or a NaN decodes to NaN throughout.
 * x_dev: dtype ZIPML_F32 or ZIPML_BF16, row-major, ldx >= cols elements between rows (rows that are
 * 16-byte aligned are read faster).  Draws: Philox as above with counter (row, col / 8, epoch * 256 + 16 +
 * tag), output word (col % 8) / 2, its low half for even columns, its high half for odd ones; tag in 0..239
 * tells the tensors of one step apart.  Asynchronous. */
int zipml_act_encode(void *stream, const void *x_dev, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                     uint64_t seed, uint32_t epoch, int tag, void *act_dev);

/* The values that act_dev stands for, in out_dev[rows][ldo], ldo >= cols.  Asynchronous. */
int zipml_act_decode(void *stream, const void *act_dev, int64_t rows, int64_t cols, void *out_dev, int dtype,
                     int64_t ldo);

/* Weight gradient of a linear layer Y = X W^T from its stored input:
 *   dW[o][i] = sum_t dY[t][o] Q(X)[t][i],   or dW += that with ZIPML_WGRAD_ADD,
 * the estimator of eq. (5) for a layer: unbiased, as Q's draws are independent of dY given X.  dY_dev: rows x d_out,
 * lddy >= d_out; act_dev: rows x d_in as zipml_act_encode wrote it; dw_dev: fp32, d_out rows of d_in values, lddw >=
 * d_in apart.  Products are exact (fp32 dY is taken as three bf16 terms, which hold values of 2^-110 and more exactly and smaller ones
 * to 2^-133; a bf16 dY is taken as it is), sums are in fp32, in an order that depends on
 * the sizes alone: the same call gives the same bits.  A NaN group of X makes its columns of dW NaN.  d_out and d_in
 * up to 2^24.  Asynchronous. */
#define ZIPML_WGRAD_ADD 1
size_t zipml_act_wgrad_workspace_bytes(int64_t rows, int64_t d_out, int64_t d_in, int dtype);
int zipml_act_wgrad(void *stream, const void *dy_dev, int dtype, int64_t lddy, const void *act_dev, int64_t rows,
                    int64_t d_out, int64_t d_in, int flags, float *dw_dev, int64_t lddw, void *workspace_dev,
                    size_t workspace_bytes);

/* Gated linear recurrence over packed sequences:
 *   f_t = sigmoid(z_t),  h_t = f_t h_{t-1} + (1 - f_t) x_t,  y_t = h_t,  channel by channel, states in fp32.
 * x_dev, z_dev, y_dev: tokens x channels, dtype ZIPML_F32 or ZIPML_BF16, rows ld* >= channels apart (so x and z may be
 * two halves of one projection, the second of which begins at a multiple of 8 bf16 or 4 fp32 values: the first value of each
 * tensor has to be 16-byte aligned, as everywhere, its rows need not be).  seq_start_dev: n_seq + 1 ascending offsets; sequence s
 * holds the tokens from seq_start[s] up to seq_start[s + 1], none if they are equal; NULL with n_seq = 1: all tokens are one sequence.
 * Tokens in no sequence (before the first offset, from the last one on) give y = 0.  Offsets that do not ascend or lie
 * outside the tokens give undefined results, but nothing outside the arrays is touched.  Outputs must not overlap inputs.
 * h0_dev [n_seq][channels]: the states before the sequences, NULL for zeros.  h_last_dev [n_seq][channels], optional:
 * the states after them (an empty sequence hands its h0 on).  A NaN or an infinity stays within its sequence and channel.
 * Gates that are nearly open cost no accuracy: what a state forgets is held to a few units of 2^-24 of itself, and a state is
 * rounded to fp32 a few times a block of ZIPML_SCAN_BLOCK tokens, not at every token.
 * For training, act_x_dev, act_z_dev (zipml_act_bytes(tokens, channels) bytes each) and states_dev
 * ([ceil(tokens / ZIPML_SCAN_BLOCK)][channels], the state before each block of so many tokens) are written for
 * zipml_scan_backward: x as zipml_act_encode stores it with `tag`, z clamped to [-16, 16] and stored with tag + 1
 * (tag in 0..238).  For serving all three are NULL.  Asynchronous. */
#define ZIPML_SCAN_BLOCK 256
size_t zipml_scan_workspace_bytes(int64_t tokens, int64_t channels);
int zipml_scan_forward(void *stream, const void *x_dev, int64_t ldx, const void *z_dev, int64_t ldz, int dtype,
                       int64_t tokens, int64_t channels, const int64_t *seq_start_dev, int64_t n_seq,
                       const float *h0_dev, void *y_dev, int64_t ldy, float *h_last_dev, void *act_x_dev,
                       void *act_z_dev, float *states_dev, uint64_t seed, uint32_t epoch, int tag,
                       void *workspace_dev, size_t workspace_bytes);

/* Backward pass of zipml_scan_forward from its stored inputs Q(x), Q(z):
 *   d_t = dy_t + f_{t+1} d_{t+1}  (a sequence's last token: dy_t + dh_last),
 *   dx_t = (1 - f_t) d_t,  dz_t = d_t (h_{t-1} - Q(x_t)) f_t (1 - f_t),  dh0 = f d of its first token,
 * with f = sigmoid(Q(z)) and the states formed again from Q(x), Q(z): from h0 at a sequence's start and from states_dev
 * at the start of each block of ZIPML_SCAN_BLOCK tokens.  dy, dx, dz: dtype, any rows apart; dh_last_dev (NULL for zeros)
 * and dh0_dev (optional): [n_seq][channels].  Tokens in no sequence give dx = dz = 0; an empty sequence's dh0 is its
 * dh_last.  seq_start_dev, n_seq, h0_dev and the sizes as in the forward pass.  Outputs must not overlap inputs: dy is read twice.
 * x and z are stored 32 channels to a step, so a NaN or an infinity of x (a NaN of z) in one channel reaches the 32 of its group: dz
 * of that token and, through the states, of later ones up to the end of the block of ZIPML_SCAN_BLOCK (in its own channel up to the
 * sequence's end); z's also dx and dz of that token and of all earlier ones of its sequence, and dh0.  Asynchronous. */
int zipml_scan_backward(void *stream, const void *act_x_dev, const void *act_z_dev, const float *states_dev,
                        const void *dy_dev, int64_t lddy, int dtype, int64_t tokens, int64_t channels,
                        const int64_t *seq_start_dev, int64_t n_seq, const float *h0_dev,
                        const float *dh_last_dev, void *dx_dev, int64_t lddx, void *dz_dev, int64_t lddz,
                        float *dh0_dev, void *workspace_dev, size_t workspace_bytes);

/* Waits for the stream and returns the status word that the last zipml_scan_forward or zipml_scan_backward left in this workspace:
 * ZIPML_OK or ZIPML_ETIMEOUT.  Blocks of a call wait for the states that enter them; blocks that a block waits for always run, but
 * no wait lasts longer than some seconds (ZIPML_KNOB_SPIN_LIMIT): past that what depends on it is NaN and the status says so. */
int zipml_scan_status(void *stream, const void *workspace_dev, size_t workspace_bytes);

/* One token of each of `rows` requests (serving): row r takes the state in row slots[r] of h_dev [n_slots][channels]
 * (row r without slots_dev) one step on, in place, and y gets it.  A row whose slot is outside 0..n_slots - 1 belongs to no
 * request: y = 0, no state is touched.  No two rows may name the same slot.  The state is rounded to fp32 at every token, so what
 * a token changes in it by less than 2^-25 of it (1 - f < 2^-25: z > 17.3) is lost.  Asynchronous. */
int zipml_scan_step(void *stream, const void *x_dev, int64_t ldx, const void *z_dev, int64_t ldz, int dtype,
                    int64_t rows, int64_t channels, float *h_dev, int64_t n_slots, const int32_t *slots_dev,
                    void *y_dev, int64_t ldy);

/* ---- layers whose product runs on 8-bit codes -------------------------------------------------
 * Rows (of tokens, or of a weight matrix, one for each output) as 8-bit codes with one scale a row, what makes such rows (an
 * encoder, the norm in front of a layer), the product of two sets of them, and the norm's backward pass; and the norm of all
 * gradients of a step.  All calls are asynchronous and may be captured in a graph.  Workspaces as above: no preparation, shared by
 * calls that follow one another on a stream.  Vectors (scales, gain, bias, rstd, dgain) need be aligned to their type only, so that
 * calls may take part of the rows, and parameters lie side by side.  Outputs must not overlap inputs except where it is said.
 *
 * Form of the codes (public): int8, rows ldc bytes apart, a multiple of 16 and at least cols; the bytes of a row from cols up to the
 * next multiple of 16 are zeros (encoders write them).  value = code * scale of the row, fp32.
 *   scale = max(max |v| / 127, 2^-126),  t = v * (1 / scale),  each a single fp32 operation;
 *   ZIPML_NEAREST: code = t rounded to an integer, ties to even;
 *   ZIPML_STOCHASTIC: code = floor(t + (k + 1/2) / 2^16), at most 127 in magnitude, k a 16-bit draw: v in expectation, to 2^-17 of
 *   the scale.  Draws as those of zipml_act_encode, from (seed, epoch, tag, row, column).
 * A row that holds an infinity or a NaN has a scale of NaN and codes of zero: all it is multiplied with becomes NaN.  (The largest
 * number of fp32 itself decodes to an infinity: 127 times its scale rounds to 2^128; the one below it does not.) */
#define ZIPML_NEAREST    0
#define ZIPML_STOCHASTIC 1
int zipml_row8_encode(void *stream, const void *x_dev, int dtype, int64_t rows, int64_t cols, int64_t ldx, int rounding,
                      uint64_t seed, uint32_t epoch, int tag, void *codes_dev, int64_t ldc, float *scales_dev);

/* The values that the codes stand for, rounded to dtype once. */
int zipml_row8_decode(void *stream, const void *codes_dev, int64_t ldc, const float *scales_dev, int64_t rows, int64_t cols,
                      void *out_dev, int dtype, int64_t ldo);

/* Linear layer on codes: y[t][o] = ((sum_i x[t][i] w[o][i]) * x_scales[t]) * w_scales[o] + bias[o]: the sum is exact (32-bit
 * integers), what follows is in fp32 and rounded to dtype once.  x_dev: codes of `rows` tokens, w_dev: of d_out rows of weights,
 * both d_in wide, rows at most 4 MiB apart; bias_dev NULL: none.  d_in up to 131,071 (ZIPML_ERANGE beyond: the sum could leave 32
 * bits), d_out up to 2^24.  A row with a scale of NaN gives NaN.  The same call with rows of a gradient, encoded by draws, and the
 * codes of W^T gives the layer's input gradient, unbiased as those draws are independent of W's codes.
 * rows up to 2^31, rows * d_out up to 2^40.  Workspace: the bytes with which the call is fastest; they fall and rise with the number of
 * rows.  256 are enough for every call (ZIPML_EWORKSPACE below): with less than is asked for the contraction is not cut into as many
 * ranges, which may take longer and changes no bit.  So one workspace may serve calls of any sizes: the largest of theirs is best. */
size_t zipml_row8_product_workspace_bytes(int64_t rows, int64_t d_out, int64_t d_in);
int zipml_row8_product(void *stream, const void *x_dev, int64_t ldx, const float *x_scales_dev, const void *w_dev, int64_t ldw,
                       const float *w_scales_dev, const float *bias_dev, int64_t rows, int64_t d_out, int64_t d_in, void *y_dev,
                       int dtype, int64_t ldy, void *workspace_dev, size_t workspace_bytes);

/* Root-mean-square norm of a residual stream:
 *   r = x + add, formed in fp32 and rounded to dtype (x alone without add_dev),  rstd = 1 / sqrt(mean r^2 + eps),  v = (r * rstd) * gain,
 * row by row; mean and root in 64 bits, rstd rounded to fp32 once.  Outputs, each of them optional but one of the first two:
 * y_dev, v rounded to dtype; codes_dev with scales_dev, v as 8-bit codes (ZIPML_NEAREST); sum_dev, r (for the next block's residual
 * and the backward pass); rstd_dev, fp32 [rows] (for the backward pass).  x, add, sum, y: dtype, rows ld* >= cols apart, each one's
 * leading dimension ignored where it is NULL; gain_dev: fp32 [cols], NULL for ones; eps finite and not negative
 * (with 0 a row of zeros gives NaN, as the formula has it).  sum_dev or y_dev
 * may be x_dev or add_dev themselves (with the same leading dimension); otherwise outputs must not overlap inputs. */
int zipml_norm_forward(void *stream, const void *x_dev, int64_t ldx, const void *add_dev, int64_t ldadd, int dtype, int64_t rows,
                       int64_t cols, const float *gain_dev, float eps, void *sum_dev, int64_t ldsum, void *y_dev, int64_t ldy,
                       void *codes_dev, int64_t ldc, float *scales_dev, float *rstd_dev);

/* Its backward pass, from the r and rstd that it kept: with n = r * rstd and a = dy * gain,
 *   dx = dsum + rstd (a - n mean(a n)),  the gradient of x and of add alike,    dgain = sum over the rows of dy n,
 * dgain (fp32 [cols], NULL if it is not wanted) in an order of the sizes alone, or added to what is there with ZIPML_NORM_ADD.
 * dsum_dev: the gradient that reaches r by the residual stream, NULL for none.  dx_dev may be dy_dev, sum_dev or dsum_dev itself.
 * The workspace is for dgain: NULL will do without. */
#define ZIPML_NORM_ADD 1
size_t zipml_norm_backward_workspace_bytes(int64_t rows, int64_t cols);
int zipml_norm_backward(void *stream, const void *dy_dev, int64_t lddy, const void *sum_dev, int64_t ldsum, int dtype, int64_t rows,
                        int64_t cols, const float *gain_dev, const float *rstd_dev, const void *dsum_dev, int64_t lddsum,
                        void *dx_dev, int64_t lddx, float *dgain_dev, int flags, void *workspace_dev, size_t workspace_bytes);

/* Global norm of the gradients of a step, and the gradients scaled down to it:
 *   norm = sqrt(sum of all g^2),  factor = 1 where norm <= max_norm, else max_norm / norm,  out = factor * g rounded to its type.
 * tensors_host: n_tensors (1 .. 2^20) descriptions, read before the call returns (a captured graph keeps the addresses in them).
 * Gradients and outputs are aligned to their types; out_dev may be grad_dev itself (of the same type) or NULL where only the norm
 * is wanted; no output may overlap another output or another tensor's gradient.  norm_dev gets {norm, factor}.  Squares are summed
 * in 64 bits in an order of the sizes alone.  max_norm may be infinite: gradients are measured and copied, not scaled.  A norm that is
 * not finite leaves nothing hidden: an infinity gives factor 0 (and NaN where it stands) or, with an infinite max_norm, stays as it is;
 * a NaN makes all outputs NaN. */
typedef struct {
    const void *grad_dev;
    void *out_dev;
    int64_t count;               /* values, 0 .. 2^33 */
    int32_t grad_dtype, out_dtype;
} zipml_clip_tensor;
size_t zipml_clip_workspace_bytes(int64_t n_tensors);
int zipml_clip(void *stream, const zipml_clip_tensor *tensors_host, int64_t n_tensors, float max_norm, float *norm_dev,
               void *workspace_dev, size_t workspace_bytes);

/* ---- parity / debug exports (not on the timed path) --------------------------------------- */

/* Canonical codes of one packed copy (`copy` = 1 or 2): codes_dev[n][d], row-major uint8. */
int zipml_unpack_codes(void *stream, const void *packed_dev, int copy, int64_t n, int64_t d,
                       int bits, uint8_t *codes_dev);

/* Runs the single step `step` of the epoch from the model in x_dev (updated in place) and exposes
 * its intermediates; any output pointer may be NULL.  model_codes_dev[d] and grad_codes_dev[d] are
 * the signed integer codes of Q3 / Q4, acc_dev[batch] the int32 dot products (integer mode only),
 * r_dev[batch] the residuals Q2(a_i)^T x - b_i, g_dev[d] the mean gradient before Q4.
 * Without flags the step runs in a launch of its own kind (the vector loop).  With
 * ZIPML_SGD_PRODUCTION it runs in the persistent launch and on the step loop that zipml_sgd_epoch
 * uses: one of the two matrix-core loops for evenly spaced 2-, 4- or 8-bit levels, batch a multiple
 * of 64, an fp32 model and more than one workgroup (only r_dev and g_dev may be asked for then,
 * ZIPML_EINVAL otherwise), or the end-to-end loop for model_bits > 0 on more than one workgroup
 * (all five outputs).  Other shapes return ZIPML_EUNSUPPORTED (other level tables through
 * zipml_sgd_status, with x_dev left untouched). */
int zipml_debug_step(void *stream, const void *packed1_dev, const void *packed2_dev,
                     const float *levels_dev, const uint16_t *grid_idx_dev, float grid_lo,
                     float grid_step, int grid_max, const float *b_dev, int64_t n, int64_t d,
                     int bits, float *x_dev, int64_t batch, float lr, int grad_bits,
                     int model_bits, uint64_t seed, uint32_t epoch, int64_t step, int flags,
                     int32_t *model_codes_dev, int32_t *acc_dev, float *r_dev, float *g_dev,
                     int32_t *grad_codes_dev, void *workspace_dev, size_t workspace_bytes);

/* What zipml_row8_product does for these sizes and a workspace of this size: its tiles (outputs x tokens, shared by `waves` waves of 64 threads), in how many ranges
 * it takes the contraction (joined by a second launch), whether results are written past the caches (for y at the start of a line of
 * 128 bytes), and the workgroups of its (first) launch.  Runs on the host. */
typedef struct {
    int32_t outputs, tokens, waves, ranges, past_caches;
    int64_t workgroups;
} zipml_product_plan;
int zipml_debug_product_plan(int64_t rows, int64_t d_out, int64_t d_in, int dtype, int64_t ldy, size_t workspace_bytes,
                             zipml_product_plan *plan_host);

/* A plain streaming pass of known size, for measurements: reads `bytes` bytes (a multiple of 16)
 * at src_dev once, XORs all their 32-bit words into *sink_dev (which the caller clears beforehand)
 * and, if dst_dev is not NULL, also stores them there (a copy).  Asynchronous.  It gives the
 * streaming-read rate of the machine for a roofline, and a launch whose HBM traffic is known, by
 * which hardware byte counters can be scaled. */
int zipml_debug_stream(void *stream, const void *src_dev, void *dst_dev, size_t bytes,
                       uint32_t *sink_dev);

/* Development knobs: process-wide overrides of choices the library otherwise makes by itself, for
 * sweeps, A/B measurements and tests that steer kernel selection (the library never reads the
 * environment).  value = -1 restores the automatic choice.  Values out of a knob's range are
 * ignored by the code that consults it.  Returns ZIPML_EINVAL for an unknown knob. */
#define ZIPML_KNOB_TARGET_WORKGROUPS 0  /* most feature-owner workgroups wanted (default: by sizes; without
                                            effect on epochs on even levels with one exchange a step, at up
                                            to 1,024 samples and 16,384 features: 64 features to each)    */
#define ZIPML_KNOB_NO_MATRIX_CORES   1  /* 1: evenly spaced levels stay on the vector-ALU step loop    */
#define ZIPML_KNOB_CHUNK_SAMPLES     2  /* chunk size of minibatches taken in chunks                    */
#define ZIPML_KNOB_MAX_REPLICAS      3  /* most replicas of the workgroups that share the chunks        */
#define ZIPML_KNOB_ROWS_MIN_BATCH    4  /* smallest minibatch for the sample-owner kernel (>= 16384)    */
#define ZIPML_KNOB_ROWS_ITEM_BLOCKS  5  /* 64-feature blocks per wave and item of that kernel (at 2 bits any
                                            value keeps the integer kernel; 101, 102: the 4-bit floating-point
                                            dot pass with tiles of 64, 128 samples)                      */
#define ZIPML_KNOB_ROWS_WORKGROUPS   6  /* its number of workgroups                                     */
#define ZIPML_KNOB_SPIN_LIMIT        7  /* polls before a device-wide wait or a recurrence's gives up
                                            (0: at once)                                              */
#define ZIPML_KNOB_HOST_DP           8  /* 1: the dynamic program of zipml_levels runs on the host     */
#define ZIPML_KNOB_HIST_FEATURES     9  /* features per workgroup of the bin-moment kernel              */
#define ZIPML_KNOB_STORE_EXCHANGE_MIN 10 /* smallest (workgroups x samples of one exchange) from which
                                            the sums travel through tagged stores and reducer
                                            workgroups instead of atomics (0: wherever the loop can; a
                                            huge value: never; by itself the library asks for 32768
                                            and at least 128 workgroups).  Any value keeps epochs on
                                            even levels on the loop that can exchange so, which by
                                            itself has minibatches in chunks, two code pairs and more
                                            than 16,384 features                                   */
#define ZIPML_KNOB_COOPERATIVE_LAUNCH 11 /* 1: the epoch kernels go through the runtime's cooperative
                                            launch (it checks that the grid can be resident, as the
                                            library does itself, and queues such launches apart from
                                            the stream's other work: some 20 us per call)          */
#define ZIPML_KNOB_REDUCER_WORKGROUPS 12 /* workgroups that only reduce the tagged partial sums, on
                                            compute units the launch leaves idle (0: none; 100 + n: n
                                            of them with pieces of four words instead of eight)   */
#define ZIPML_KNOB_PREFETCH_WORKGROUPS 13 /* workgroups that only read the packed codes of a later chunk
                                            into the cache, on compute units still idle (0: none)  */
#define ZIPML_KNOB_COUNT            14
int zipml_debug_set(int knob, int64_t value);

#ifdef __cplusplus
}
#endif
#endif /* ZIPML_H */
