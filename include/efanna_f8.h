/*
 * Matrices in 8-bit floating point with a scale for each block of 128, and what a linear layer is
 * trained and served with in them: the inputs that its backward pass needs kept in 8 bits, its
 * weights both ways round, products, and the gradient of the weights.
 *
 * Part of the library that efanna.h describes; statuses, streams and element types are those.
 *
 * Format.  Coordinates of a row in blocks of 128, nb = ceil(d / 128) of them, the last one filled up
 * with zeros.  A block holds a scale byte b, which stands for 2^(b - 127) (255: NaN), and 128 codes:
 *   EFANNA_E4M3  sign, 4 exponent bits (bias 7), 3 of mantissa: up to 448; 0x7F and 0xFF are NaN
 *   EFANNA_E5M2  sign, 5 exponent bits (bias 15), 2 of mantissa: up to 57344; 0x7C and 0xFC are
 *                infinities, above them NaN
 *   codes  n * 128 * nb bytes, 16-byte aligned.
 *   scales n * sp bytes, sp = nb rounded up to a multiple of 4, 4-byte aligned; padding bytes 0.
 * A value is code * scale, exactly; one of 2^128 (which the largest float32 numbers are rounded to) reads
 * as an infinity in every type, and is one in gradients and in products to float32 (products to 16 bits take
 * it as 2^128).
 * 1 <= d <= EFANNA_F8_MAX_D, n < 2^31 - 65536.  Row counts may be 0 (pointers to what has no elements
 * may be NULL).  Element types of other matrices: EFANNA_F32, EFANNA_F16 or EFANNA_BF16, aligned to
 * their size.  All calls are asynchronous on `stream`, can be captured into a graph, and allocate
 * nothing; calls that may run at the same time need workspaces of their own.
 */
#ifndef EFANNA_F8_H
#define EFANNA_F8_H

#include "efanna.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EFANNA_F8_MAX_D 65536
#define EFANNA_F8_MAX_LDY 16777216   /* elements between the rows of a gradient: fewer */
#define EFANNA_E4M3 0
#define EFANNA_E5M2 1

/* Rows of X [device] (n rows of d elements of type dtype, ldx >= d elements apart) to a table.
 * A block's scale is the smallest power of two, 2^-127 at least, that leaves none of its finite magnitudes
 * beyond the largest code (a block of zeros has 2^-127); a code is the nearest value to x / scale, ties to the even
 * code.  A NaN becomes a NaN; an infinity an infinity in E5M2 and a NaN in E4M3; the block's other
 * coordinates are held as if it were not there. */
int efanna_f8_quantise(const void *X, int32_t dtype, int64_t n, int32_t d, int64_t ldx, int32_t format,
                       uint8_t *codes, uint8_t *scales, void *stream);

/* A matrix W (n rows of d elements, ldw apart, n <= EFANNA_F8_MAX_D) to its table and, where t_codes is not
 * NULL, to the table of its transpose (d rows of n), with one scale for each tile of 128 x 128, so
 * that both hold the same values. */
int efanna_f8_weights(const void *W, int32_t dtype, int32_t n, int32_t d, int64_t ldw, int32_t format,
                      uint8_t *codes, uint8_t *scales, uint8_t *t_codes, uint8_t *t_scales, void *stream);

/* Rows of a table by id: out[i] = factor * row ids[i], m rows of d elements, dense.
 * ids    [device] m int32, or NULL: rows 0 .. m - 1 (m <= n).  An id below 0 or of n and more names an
 *        empty slot: a row of zeros.
 * Values are multiplied in float32 and rounded once (to nearest, ties to even). */
int efanna_f8_rows(const uint8_t *codes, const uint8_t *scales, int32_t format, int64_t n, int32_t d,
                   const int32_t *ids, int64_t m, float factor, int32_t dtype, void *out, void *stream);

/* out[i * ldo + j] = a_i . b_j for the m rows of one table and the n rows of another, ldo >= n; the tables may
 * differ in their format.  Sums are held in float32 and rounded once to dtype.
 * For EFANNA_F32 every product and sum is one of float32 at least (values below 2^-126 count in steps of
 * 2^-133).  For 16-bit results the matrix units take 8-bit operands, whose products they add in groups of eight,
 * each product cut off at 2^-14 of its group's largest: at most 2^-11 of the sum of magnitudes is lost.  Of sums of
 * a thousand and more random terms two to three in a hundred were then a step of their type beside the nearest
 * number, and the error against exact sums 0.2 % larger at most; sums of terms of one sign came out smaller by 3e-6
 * of them, of terms of very different size by 1e-4.  Sums whose terms cancel are better taken to EFANNA_F32 and
 * converted.
 * ws     [device] 256-byte aligned, efanna_f8_product_workspace_bytes bytes; may be NULL where that is 0.
 * EFANNA_EUNSUPPORTED for what one launch does not take: 2^23 tiles of 256 x 256 and more (half a terabyte of
 * output). */
size_t efanna_f8_product_workspace_bytes(int64_t m, int64_t n, int32_t d, int32_t dtype);

int efanna_f8_product(const uint8_t *a_codes, const uint8_t *a_scales, int32_t a_format, int64_t m,
                      const uint8_t *b_codes, const uint8_t *b_scales, int32_t b_format, int64_t n, int32_t d,
                      int32_t dtype, void *out, int64_t ldo, void *ws, size_t ws_bytes, void *stream);

/* out[j * ldo + c] = sum over t of dY[t * ldy + j] * row t of a table [c]: the gradient of a layer's weights from that
 * of its output (m rows of n elements of type dtype, ldy >= n apart) and its input as held (m rows of d
 * coordinates).  ldo >= d; n <= EFANNA_F8_MAX_D; with m = 0 the sums are zeros.
 * Nothing is rounded but sums, in float32, and the result, to out_dtype (values of the table below 2^-126 count
 * in steps of 2^-133, those of dY are taken in parts, of which the ones below 2^-133 are lost).
 * EFANNA_EUNSUPPORTED for ldy >= EFANNA_F8_MAX_LDY.
 * ws     [device] 256-byte aligned, efanna_f8_gradient_workspace_bytes bytes; may be NULL where that is 0. */
size_t efanna_f8_gradient_workspace_bytes(int64_t m, int32_t n, int32_t d, int32_t dtype);

int efanna_f8_gradient(const void *dY, int32_t dtype, int64_t m, int32_t n, int64_t ldy, const uint8_t *codes,
                       const uint8_t *scales, int32_t format, int32_t d, int32_t out_dtype, void *out,
                       int64_t ldo, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EFANNA_F8_H */
