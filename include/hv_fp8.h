/*
 * hv_fp8.h -- operators that make and read weights held in 8 bits.
 *
 * The paper's threat model asks that the bytes that were checked are the bytes
 * that are used (Problem Statement & Threat Model: the TOCTOU discussion), and
 * its loader runs the model it has verified.  These operators run a decoder's
 * projections on 8-bit weights as they lie in memory when the calls of hv.h hash
 * them: codes and scales, with no second copy in another layout.  (That goes for
 * weights whose rows are 16-byte aligned.  Rows at other addresses hv_fp8_matmul may
 * copy to its workspace, anew in each call, and multiply from there.)
 * Held in 8 bits, a weight set also takes half the time to hash.
 *
 * Format.  A code is an 8-bit floating-point number, OCP E4M3 (1 sign, 4
 * exponent and 3 mantissa bits, largest value 448, NaN 0x7f and 0xff, no
 * infinity).  A matrix [rows][cols] of codes comes with 32-bit scales, one for
 * every group of
 *   - 128 consecutive columns of one row (activations): scales
 *     [rows][ceil(cols / 128)], or
 *   - 128 columns of 128 consecutive rows (weights): scales
 *     [ceil(rows / 128)][ceil(cols / 128)];
 * the last group of a row, and the last rows' groups, are shorter where the
 * sizes are no multiples of 128.  Scales are contiguous.  The value of a code is
 * the code's number times its group's scale.
 *
 * Quantisation.  A group's scale is max|y| / 448 over its finite values, at
 * least 2^-126, and 1 where that maximum is 0.  A value's code is y / scale in 32
 * bits, rounded to the nearest E4M3 number, ties to even.  A NaN or an infinity
 * becomes a NaN code and leaves the rest of its group alone.
 *
 * Every call is asynchronous on `stream`: it queues kernels only (no upload, no
 * host wait, no allocation, no memset), so it may be captured in a HIP graph.
 * All pointers are device pointers of the device that is current.  Leading
 * dimensions (ld_*) count elements between the starts of consecutive rows and are
 * at least the columns of a row.  Rows need no alignment beyond that of their
 * element type; 16-byte aligned ones are read faster.  Inputs and outputs must not
 * overlap, but for the case that hv_fp8_rms_norm names.  A call with no elements to
 * write does nothing.
 * Results do not depend on the stream or on what runs beside, and are equal bit
 * for bit from call to call.
 *
 * Common errors: HV_ERR_INVALID_ARG for an unknown type, a NULL or misaligned
 * pointer where elements are read or written, a leading dimension below the
 * columns, or sizes past the limits (rows 2^31 - 1, columns 2^24, leading
 * dimensions 2^31); HV_ERR_HIP.
 */
#ifndef HV_FP8_H
#define HV_FP8_H

#include "hv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the wider matrices. */
typedef int32_t hv_type;
#define HV_BF16 0 /* bfloat16 */
#define HV_F16 1  /* IEEE half */
#define HV_F32 2  /* IEEE single */

/* Codes and scales of x [rows][cols].
 *   tile_rows: rows that share a scale, 1 (activations) or 128 (weights).
 *   codes: [rows][cols]; scales: [ceil(rows / tile_rows)][ceil(cols / 128)].
 * Errors: HV_ERR_INVALID_ARG also for another tile_rows. */
hv_status hv_fp8_quantize(hv_type type, const void* x, uint64_t ld_x, uint64_t rows, uint64_t cols,
                          uint32_t tile_rows, uint8_t* codes, uint64_t ld_codes, float* scales, hipStream_t stream);

/* Root-mean-square norm with the residual's addition, quantised by rows:
 *   h = x + residual;  y = h / sqrt(mean(h^2) + eps) * weight;
 * the mean is over a row's columns.  The sum h, its squares and y are formed in
 * 32 bits; y is quantised from there, and h is also rounded to the type and
 * written to residual_out, the residual of the next layer.
 *   residual, residual_out: [rows][cols] of the type; both NULL for h = x.
 *                           residual_out may be x or residual itself (same
 *                           address and leading dimension).
 *   weight: [cols] of the type.
 *   codes: [rows][cols]; scales: [rows][ceil(cols / 128)].
 * Errors: HV_ERR_INVALID_ARG also where only one of residual and residual_out
 * is NULL, or eps is negative or NaN. */
hv_status hv_fp8_rms_norm(hv_type type, const void* x, uint64_t ld_x, const void* residual, uint64_t ld_residual,
                          const void* weight, float eps, uint64_t rows, uint64_t cols, void* residual_out,
                          uint64_t ld_residual_out, uint8_t* codes, uint64_t ld_codes, float* scales,
                          hipStream_t stream);

/* silu(gate) * up, quantised by rows: y = gate / (1 + exp(-gate)) * up in 32 bits,
 * and gate * exp(gate) * up for gates below -87, where exp(-gate) leaves them.
 *   gate, up: [rows][cols] of the type; they may be the two halves of one
 *             matrix's rows.
 *   codes: [rows][cols]; scales: [rows][ceil(cols / 128)]. */
hv_status hv_fp8_gated(hv_type type, const void* gate, uint64_t ld_gate, const void* up, uint64_t ld_up,
                       uint64_t rows, uint64_t cols, uint8_t* codes, uint64_t ld_codes, float* scales,
                       hipStream_t stream);

/* Scratch bytes hv_fp8_matmul needs for a result of the type and these sizes; 0
 * where it needs none, and for a type or sizes that the call refuses.
 *   aligned: nonzero where a and b are 16-byte aligned and ld_a and ld_b multiples
 *            of 16.  An operand for which that does not hold may be copied to
 *            aligned rows there first. */
size_t hv_fp8_matmul_workspace_bytes(hv_type type, int aligned, uint64_t m, uint64_t n, uint64_t k);

/* c [m][n] = A times the transpose of B, for A [m][k] with scales by rows and B
 * [n][k] with scales by blocks:
 *   c[i][j] = sum over groups g of a_scales[i][g] * b_scales[j / 128][g] *
 *             (sum over the group's columns t of a[i][t] * b[j][t]).
 * Accumulators have 32 bits and c is rounded once, to the type.  For HV_F32 all
 * products and sums are in 32 bits.
 * For the 16-bit types the matrix unit adds the products of 16 neighbouring
 * columns in fixed point and drops what is below 2^-13 of the largest of them.  Each
 * 16 are then off by up to 15 * 2^-13 of their largest product, c by the sum of that
 * (times the scales): at worst 1.8e-3 of the sum of the terms' magnitudes, which
 * is not relative to c where large terms cancel.  Measured, as a whole: 1.4e-5 of c for
 * ordinary codes, 3.5e-5 where 0.2% of A's columns are 30 times the others, 6.5e-5
 * where they are 300 times, beside roundings to the type of 2.1e-4 (HV_F16) and
 * 1.7e-3 (HV_BF16); a single c near zero can lose more than its rounding.  Who needs
 * 32-bit sums takes HV_F32, at half the matrix unit's rate, and rounds.
 * k = 0 gives zeros.  The product of any two scales that meet is formed in 32 bits:
 * it has to be finite, below 2^-126 it has fewer bits, and from 2^-150 down it is zero.
 *   c: [m][n] of the type, with leading dimension ld_c.
 *   workspace: >= hv_fp8_matmul_workspace_bytes(...), 256-byte aligned; NULL where
 *              that is 0, or where ld_a or ld_b is 2^23 or more.  Scratch: calls that
 *              share one must share a stream.
 * Errors: HV_ERR_INVALID_ARG also for m or n above 2^27; HV_ERR_WORKSPACE for a
 * missing, short or misaligned workspace. */
hv_status hv_fp8_matmul(hv_type type, const uint8_t* a, uint64_t ld_a, const float* a_scales, const uint8_t* b,
                        uint64_t ld_b, const float* b_scales, uint64_t m, uint64_t n, uint64_t k, void* c,
                        uint64_t ld_c, void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HV_FP8_H */
