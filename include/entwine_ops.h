/*
 * entwine_ops.h - operators beside the fused GEMM-ReduceScatter of entwine.h: the row-parallel layer's product in
 * 8-bit integers (serving) and its form with experts (tokens sorted by expert, and back with weights applied).
 * The conventions of entwine.h hold: every function returns ENTWINE_OK or a negative ENTWINE_ERR_* code, nothing
 * throws, nothing allocates, nothing synchronises (but entwine_ops_status and entwine_ops_failed_waits), `stream` is a cudaStream_t passed as
 * void* (NULL = the default stream), and device pointers belong to the current device.
 *
 * These calls have no plan: each is complete in itself, keeps nothing from one call for the next, and needs no
 * workspace.  Any of them may be captured into a CUDA graph (its first call too), and calls on different streams
 * may overlap as far as their buffers allow.  Outputs must not overlap inputs or each other.  The same inputs give the
 * same bits on every call.
 *
 * Matrices are row-major; ld* is the distance between two rows in elements, at least the row's length.  Element
 * pointers need the alignment of their element only, except where a function says more; rows that start on
 * 16-byte boundaries are the fastest (K or H need not fill them).  Contiguous rows of an odd number of 16-bit elements
 * cost the dispatch a tenth more, the return, its gradients and the quantiser about twice as much.
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
                                         value-th block of 128 elements of K (counted within the CTA's share of K),
                                         which is not loaded; -1: none (default)                                       */
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

#ifdef __cplusplus
}
#endif
#endif /* ENTWINE_OPS_H_ */
