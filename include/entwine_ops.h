/*
 * entwine_ops.h - operators beside the fused GEMM-ReduceScatter of entwine.h: the row-parallel layer's product in
 * 8-bit integers and in 4-bit floats (serving), its form with experts (tokens sorted by expert, and back with weights
 * applied), and what follows its ReduceScatter in training: dropout, residual and layer norm, with their gradients.
 * The conventions of entwine.h hold: every function returns ENTWINE_OK or a negative ENTWINE_ERR_* code, nothing
 * throws, nothing allocates, nothing synchronises (but entwine_ops_status and entwine_ops_failed_waits), `stream` is a cudaStream_t passed as
 * void* (NULL = the default stream), and device pointers belong to the current device.
 *
 * These calls have no plan: each is complete in itself, keeps nothing from one call for the next, and needs no
 * workspace (but entwine_layer_norm_bwd, whose caller brings it).  Any of them may be captured into a CUDA graph (its
 * first call too), and calls on different streams may overlap as far as their buffers allow.  Outputs must not overlap inputs or each other.  The same inputs give the
 * same bits on every call.
 *
 * Matrices are row-major; ld* is the distance between two rows in elements, at least the row's length.  Element
 * pointers need the alignment of their element only, except where a function says more; rows that start on
 * 16-byte boundaries are the fastest (K or H need not fill them).  Contiguous rows of an odd number of 16-bit elements
 * cost the dispatch a tenth more, dropout a third more, the return, its gradients, the quantisers, layer norm and its
 * gradients about twice as much.
 */
#ifndef ENTWINE_OPS_H_
#define ENTWINE_OPS_H_

#include "entwine.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the matrices. */
enum { ENTWINE_BF16 = 0, ENTWINE_FP16 = 1, ENTWINE_FP32 = 2, ENTWINE_I8 = 3 };

/*
 * entwine_quant_i8 - rows to 8-bit integers, each row with a scale of its own (a token's activations, or an
 * output channel's weights: both operands of entwine_gemm_i8 have this form).
 *   amax = max_k |x[m][k]|;  scale[m] = amax / 127 (fp32);  q[m][k] = rint(127 x[m][k] / amax)
 * The rounding is that of the exact quotient, ties to even, so q is the same on every implementation; it lies in
 * [-127, 127].  A row of zeros gets scale 0 and q 0; a row that holds a NaN or an infinity gets scale NaN and
 * q 0, so that what is computed from it is NaN.
 *   x      [rows, cols], dtype ENTWINE_BF16, ENTWINE_FP16 or ENTWINE_FP32
 *   q      [rows, cols] int8     scale  [rows] fp32
 * rows = 0 is allowed and does nothing; cols >= 1.  Errors: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.
 */
int entwine_quant_i8(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, void* q, int64_t ldq,
                     float* scale, void* stream);

/*
 * entwine_gemm_i8 - the row-parallel layer's product in 8-bit integers, scaled per token and per output channel:
 *   C[m][n] = scale_a[m] scale_b[n] sum_k A[m][k] B[n][k] + bias[n]
 * The int32 sum is exact, the scaling is fp32, C is rounded once.  In fp32 the order is ((sum scale_a) scale_b) + bias:
 * where |sum| scale_a passes fp32's range (a token scale of 2^97 is the least that can do it) C is infinite, whatever
 * scale_b.
 *   A [M, K] int8, B [N, K] int8 (K contiguous, as entwine.h's default layout): both 16-byte aligned with lda and
 *   ldb multiples of 16 (K itself may be any length: what follows it in a row is not read into the sum)
 *   scale_a [M], scale_b [N], bias [N] fp32; bias may be NULL
 *   C [M, N], c_dtype ENTWINE_BF16, ENTWINE_FP16 or ENTWINE_FP32
 * M = 0 is allowed and does nothing, M <= 2147418111; 1 <= N <= 2147483392; 1 <= K <= 131071 (the largest sum fits
 * int32).
 * Errors: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.  Device-side waits are bounded: see entwine_ops_status.
 */
int entwine_gemm_i8(const void* A, int64_t lda, const float* scale_a, const void* B, int64_t ldb,
                    const float* scale_b, const float* bias, void* C, int c_dtype, int64_t ldc, int64_t M, int64_t N,
                    int64_t K, void* stream);

/*
 * entwine_gemm_i8_grouped - the same product with a weight matrix per expert, for rows sorted by expert: rows
 * [offsets[g], offsets[g+1]) of A are multiplied with B[g] and scaled with scale_b[g] (and bias[g]).
 *   offsets [G+1] int32, device memory, non-decreasing, 0 <= offsets[0], offsets[G] <= M (as entwine_moe_dispatch
 *   writes them); bounds outside [0, M] are taken as the nearest inside, a decreasing pair as an empty expert
 *   (with decreasing offsets it is not said which of the overlapping rows are computed; nothing else is touched)
 *   B [G][N][K], expert_stride elements from one expert's matrix to the next (a multiple of 16)
 *   scale_b [G][N], bias [G][N] or NULL
 * Rows of C that belong to no expert are left as they were.  1 <= G <= 1024, G * N < 2^31; the rest as above.
 */
int entwine_gemm_i8_grouped(const void* A, int64_t lda, const float* scale_a, const void* B, int64_t ldb,
                            int64_t expert_stride, const float* scale_b, const float* bias, const int32_t* offsets,
                            void* C, int c_dtype, int64_t ldc, int64_t M, int64_t N, int64_t K, int64_t G,
                            void* stream);

/*
 * entwine_quant_mxf4 - rows to 4-bit floats (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with a power-of-two
 * scale for every 32 elements, as the OCP Microscaling Formats specification 1.0 has them (MXFP4); both operands of
 * entwine_gemm_mxf4 have this form.  For the elements of a block, amax their largest magnitude:
 *   e = min(max(floor(log2 amax) - 2, -127), 127);  scale byte e + 127 (e8m0)
 *   code = the e2m1 value nearest to x 2^-e, ties to the one with the even code, 6 where it is above
 * so the codes are the same on every implementation.  A code keeps its element's sign, also as -0.  A block of zeros
 * gets scale byte 0; a block that holds a NaN or an infinity gets scale byte 255, which stands for NaN, and codes 0.
 *   x      [rows, cols], dtype ENTWINE_BF16, ENTWINE_FP16 or ENTWINE_FP32
 *   q      [rows, (cols+1)/2] bytes: element 2i in the lower half of byte i, 2i+1 in the upper (zero behind an odd end)
 *   scale  [rows, (cols+31)/32] bytes; the last block of a row may be shorter
 * rows = 0 is allowed and does nothing; 1 <= cols <= 2147418111.  Errors: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.
 *
 * entwine_dequant_mxf4 - back to values: x = code * 2^(scale byte - 127), rounded once to dtype; NaN in a block of
 * scale byte 255.  (For a weight kept in 4 bits before a product of wider operands, or to see what was lost.)
 */
int entwine_quant_mxf4(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, void* q, int64_t ldq, void* scale,
                       int64_t lds, void* stream);
int entwine_dequant_mxf4(const void* q, int64_t ldq, const void* scale, int64_t lds, int64_t rows, int64_t cols, void* x,
                         int dtype, int64_t ldx, void* stream);

/*
 * entwine_gemm_mxf4 - the row-parallel layer's product of two such matrices:
 *   C[m][n] = sum_k a[m][k] b[n][k] + bias[n],  a and b the values that codes and scales stand for
 * Products are exact, sums fp32 in the tensor core, C is rounded once.  A scale byte of 255 makes the rows (of A) or
 * columns (of B) of C that it enters NaN.
 *   A [M, (K+1)/2], B [N, (K+1)/2] bytes of codes: 16-byte aligned with lda and ldb (in bytes) multiples of 16
 *   scale_a [M, (K+31)/32], scale_b [N, (K+31)/32] bytes: 4-byte aligned with ldsa and ldsb multiples of 4
 *   (what follows K in a row is not read into the sum; of an odd K the last upper half has to be zero)
 *   bias [N] fp32 or NULL     C [M, N], c_dtype ENTWINE_BF16, ENTWINE_FP16 or ENTWINE_FP32
 * M = 0 is allowed and does nothing, M <= 2147418111; 1 <= N <= 2147483392; 1 <= K <= 16777216.
 * Errors: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.  Device-side waits are bounded: see entwine_ops_status.
 *
 * entwine_gemm_mxf4_grouped - the same with a weight matrix per expert, for rows sorted by expert; offsets as in
 * entwine_gemm_i8_grouped.  B [G][N][(K+1)/2] with expert_stride bytes from one expert's matrix to the next (a multiple
 * of 16), scale_b [G][N][(K+31)/32] with scale_stride (a multiple of 4), bias [G][N] or NULL.  Rows of C that belong to
 * no expert are left as they were.  1 <= G <= 1024, G * N < 2^31.
 */
int entwine_gemm_mxf4(const void* A, int64_t lda, const void* scale_a, int64_t ldsa, const void* B, int64_t ldb,
                      const void* scale_b, int64_t ldsb, const float* bias, void* C, int c_dtype, int64_t ldc, int64_t M,
                      int64_t N, int64_t K, void* stream);
int entwine_gemm_mxf4_grouped(const void* A, int64_t lda, const void* scale_a, int64_t ldsa, const void* B, int64_t ldb,
                              int64_t expert_stride, const void* scale_b, int64_t ldsb, int64_t scale_stride,
                              const float* bias, const int32_t* offsets, void* C, int c_dtype, int64_t ldc, int64_t M,
                              int64_t N, int64_t K, int64_t G, void* stream);

/*
 * entwine_ops_status - synchronises `stream` and returns ENTWINE_ERR_TIMEOUT if bounded device-side waits of products on
 * the current device have run out since the calling host thread's last such query for this device (its first: since
 * the library was loaded), else ENTWINE_OK.  TIMEOUT does not say whose product it was: each one that this thread
 * answers for and that had not ended before its last query may have an incomplete C.  A query takes nothing from
 * other threads.  Not allowed on a capturing stream (ENTWINE_ERR_INVALID).
 *
 * entwine_ops_failed_waits - synchronises `stream` and gives the number of waits of products that have run out on the
 * current device since the library was loaded; it only grows.  A caller that keeps the number from before its calls
 * (so that several of them can share a thread) knows that they are complete if it has not changed after them.
 */
int entwine_ops_status(void* stream);
int entwine_ops_failed_waits(void* stream, uint64_t* count);

/* Settings of the process for its later calls (a captured call keeps those that it was captured with). */
enum {
  ENTWINE_OPS_OPT_WAIT_BUDGET_NS = 1, /* budget of every device-side wait of the products (default 2e9, at least 1e6) */
  ENTWINE_OPS_OPT_WITHHOLD_BLOCK = 2  /* host-side fault injection: the first tile of a product waits for its
                                         value-th block of 128 bytes of K (128 elements of 8 bits, 256 of 4; counted
                                         within the CTA's share of K), which is not loaded; -1: none (default)         */
};
/* ENTWINE_ERR_INVALID for an unknown key or a value out of range. */
int entwine_ops_set_option(int key, int64_t value);

/*
 * entwine_moe_dispatch - tokens sorted by expert.  ids [T][k] (int32, or int64 with ids64 != 0; contiguous) names
 * the k experts of each token, 0 <= id < E; any other value (-1, say) drops the assignment.  The assignments that
 * are left are ordered by expert, within an expert by t*k + j:
 *   offsets [E+1] int32    expert e owns rows [offsets[e], offsets[e+1]); offsets[E] rows in all
 *   row_of  [T][k] int32   the row of each assignment, -1 where it was dropped
 *   rows    [T*k][H]       rows[row_of[t][j]] = x[t]; rows behind offsets[E] are left as they were
 * x [T][H] of any dtype of this header.  x_scale / row_scale (both or neither): fp32 values [T] that go with the
 * tokens, row_scale[row_of[t][j]] = x_scale[t] (the scales of quantised rows).
 * An expert named twice by one token gets two rows.  1 <= E <= 1024, k >= 1, H >= 1, T*k < 2^31; T = 0 writes
 * offsets only.  Errors: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.
 */
int entwine_moe_dispatch(const void* x, int dtype, int64_t T, int64_t H, int64_t ldx, const float* x_scale,
                         const void* ids, int ids64, int64_t k, int64_t E, void* rows, int64_t ldr,
                         float* row_scale, int32_t* offsets, int32_t* row_of, void* stream);

/*
 * entwine_moe_dispatch_bwd - its gradient: dx[t] = sum_j d_rows[row_of[t][j]], summed in fp32 with j ascending
 * and rounded once; 0 for a token whose assignments were all dropped.
 *   d_rows [n_rows][H] and dx [T][H] of one dtype (ENTWINE_BF16, ENTWINE_FP16, ENTWINE_FP32)
 * Values of row_of outside [0, n_rows) count as dropped.
 */
int entwine_moe_dispatch_bwd(const void* d_rows, int dtype, int64_t n_rows, int64_t H, int64_t ldr,
                             const int32_t* row_of, int64_t T, int64_t k, void* dx, int64_t ldx, void* stream);

/*
 * entwine_moe_combine - the experts' outputs back at their tokens, weights applied:
 *   out[t] = sum_j w[t][j] y[row_of[t][j]], in fp32 with j ascending, rounded once; 0 where nothing is left.
 *   y [n_rows][H], out [T][H] of one dtype (ENTWINE_BF16, ENTWINE_FP16, ENTWINE_FP32); w [T][k] fp32; row_of as
 *   entwine_moe_dispatch writes it, values outside [0, n_rows) count as dropped (their weight is not used).
 */
int entwine_moe_combine(const void* y, int dtype, int64_t n_rows, int64_t H, int64_t ldy, const float* w,
                        const int32_t* row_of, int64_t T, int64_t k, void* out, int64_t ldo, void* stream);

/*
 * entwine_moe_combine_bwd - its gradients, for dout [T][H]:
 *   dy[row_of[t][j]] = w[t][j] dout[t];  dw[t][j] = sum_h dout[t][h] y[row_of[t][j]][h] (fp32), 0 where dropped.
 * Rows of dy that no assignment names are left as they were.  No two assignments may name the same row.
 */
int entwine_moe_combine_bwd(const void* dout, int dtype, int64_t T, int64_t H, int64_t ldo, const void* y,
                            int64_t n_rows, int64_t ldy, const float* w, const int32_t* row_of, int64_t k, void* dy,
                            int64_t lddy, float* dw, void* stream);

/*
 * entwine_dropout - out = residual + dropout(x), with a mask that is computed again where it is needed and never stored.
 * Column c of row r is kept if a 16-bit number, a function of (rng, row0 + r, c) alone, is at least t = rint(65536 p),
 * that is with probability 1 - t / 65536, and is then multiplied with 65536 / (65536 - t); else it is 0, whatever it
 * holds.  The sum with the residual is fp32, rounded once.
 *   The number: Philox4x32 with ten rounds (Salmon et al. 2011), key = seed, counter = (c / 8, row0 + r, low half of
 *   offset, high half of offset); its 32-bit words w0 .. w3 hold the numbers of eight columns, number j in half j % 2
 *   (0: the lower) of word j / 2.
 *   rng   int64 {seed, offset} in device memory, 8-byte aligned, read when the kernel runs: a captured call takes the
 *         values of its replay.  Another seed or another offset gives another mask.  NULL is allowed with p = 0.
 *   row0  number of the first row: the ranks that hold the shards of one matrix get the mask of the whole.
 *         0 <= row0, row0 + rows <= 2^32
 *   x, out [rows, cols] and residual [rows, cols] (or NULL): one dtype, ENTWINE_BF16, ENTWINE_FP16 or ENTWINE_FP32
 * 0 <= p < 1 with t <= 65535.  rows = 0 does nothing.  The gradient of x is the same call on the gradient of out, without
 * a residual.  Errors: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.
 */
int entwine_dropout(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* residual, int64_t ldr,
                    double p, const int64_t* rng, int64_t row0, void* out, int64_t ldo, void* stream);

/*
 * entwine_layer_norm - what follows the ReduceScatter of a training step, in one launch:
 *   hidden = residual + dropout(x)   (rounded to dtype; without residual and with p = 0 it is x)
 *   mean = sum_c hidden / cols;  rstd = 1 / sqrt(sum_c (hidden - mean)^2 / cols + eps);
 *   out = (hidden - mean) rstd weight + bias
 * computed in fp32 from the rounded hidden values, as entwine_gemm_rs_norm does (sums over more than 16384 columns in more bits).
 * dropout, p, rng, row0: entwine_dropout.
 *   x, residual (or NULL), hidden (NULL: not written), out: [rows, cols] of one dtype
 *   weight, bias (or NULL) [cols], both of w_dtype: dtype or ENTWINE_FP32
 *   mean, rstd [rows] fp32 (NULL: not written), what the gradients need;  eps >= 0
 * A row of equal values has variance 0 but for the rounding of its mean: with eps = 0 its out is NaN, or of the order of
 * the weight where the mean came out one rounding beside the values.  rows = 0 does nothing.
 *
 * entwine_layer_norm_bwd - its gradients for dout [rows, cols], with n = (hidden - mean) rstd and g = dout weight:
 *   dh = rstd (g - sum_c g / cols - n sum_c (g n) / cols) + dhidden
 *   dresidual = dh;  dx = dropout'(dh);  dweight = sum_r dout n;  dbias = sum_r dout
 *   dhidden    gradient that reaches hidden itself, down the residual stream (NULL: none)
 *   dresidual  NULL: not written (without dropout it is dx)
 *   dweight, dbias [cols] fp32, dbias may be NULL; of no rows they are 0
 *   work       work_floats fp32 values, at least what entwine_layer_norm_bwd_work gives for these extents; the partial
 *              sums of dweight and dbias, added in a fixed order.  Calls that may overlap (two streams, two graphs) need one each.
 * dweight and dbias are fp32 sums, so their error grows with the rows as such sums' does.  fp32 rows of 8193 to 16384 columns
 * take the time of rows that start anywhere, wherever they start.
 * mean and rstd, p, rng and row0 as in the forward call.  Errors of all three: ENTWINE_ERR_INVALID, ENTWINE_ERR_CUDA.
 */
int entwine_layer_norm(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* residual,
                       int64_t ldr, double p, const int64_t* rng, int64_t row0, const void* weight, const void* bias,
                       int w_dtype, float eps, void* hidden, int64_t ldh, void* out, int64_t ldo, float* mean, float* rstd,
                       void* stream);
int entwine_layer_norm_bwd_work(int64_t rows, int64_t cols, int64_t* floats);
int entwine_layer_norm_bwd(const void* dout, int dtype, int64_t rows, int64_t cols, int64_t ldo, const void* hidden,
                           int64_t ldh, const void* weight, int w_dtype, const float* mean, const float* rstd,
                           const void* dhidden, int64_t lddh, double p, const int64_t* rng, int64_t row0, void* dx,
                           int64_t lddx, void* dresidual, int64_t lddr, float* dweight, float* dbias, float* work,
                           int64_t work_floats, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ENTWINE_OPS_H_ */
