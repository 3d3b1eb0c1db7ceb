/*
 * peat_ops.h -- the operators of libpeat that a playback step runs beside the
 * compare: a linear layer's products in 8-bit integers or in 4-bit floating
 * point, the root-mean-square norm in front of such a layer, and the norm and the
 * clipping of a list of gradients.
 *
 * Playback FI (Alg. 1) computes a layer's forward output, its input gradient
 * and its weight gradient again at a lower precision from the recorded
 * (activation, weight, output gradient), and scores them against the golden
 * ones.  Here the lower precision is 8-bit integers with one scale for each
 * row of either operand: peat_quantize_i8 makes the operands,
 * peat_matmul_i8 multiplies them, peat_product_i8 does both.  Or it is 4-bit
 * floating point with a scale for each short block: peat_quantize_f4,
 * peat_matmul_f4, peat_product_f4.  What comes into the layer is a norm's output:
 * peat_rmsnorm makes it, rounded to 8 bits on the way, peat_rmsnorm_backward its
 * gradients.  A training step ends with the norm over all its gradient tensors,
 * by which they are clipped: peat_grad_norm and peat_grad_clip.
 *
 * The conventions of peat.h hold: device pointers unless said otherwise,
 * every call asynchronous on `stream`, errors as peat_status_t with the text
 * in peat_last_error(h), nothing thrown, one handle per host thread and its
 * calls in order on the GPU (its workspace is reused call after call).  The
 * workspace grows on demand; a call that has to grow it waits for the device, and
 * a block that is outgrown becomes half as large again, where there is room.
 * After a first call of the same sizes, types and alignment (of data and row
 * distances to 16 bytes, which the choice of a product's kernel counts in), the
 * calls of this header do not allocate.  A product of many rows takes, with M and
 * N rounded up to 256 and K to 64, 2 (M + N) K bytes, and for K above 1024 20 MB,
 * or where that is more 4 M N bytes for each of the 1, 2 or 4 parts in which K is
 * taken; operands that peat_product_i8 rounds add a byte for each element.
 * An operand of R rows and k along the product's axis that peat_product_f4 rounds
 * takes R (k / 2) bytes for its codes (k rounded up to whole blocks, k / 2 to 16
 * bytes), peat_f4_scale_bytes for its block scales, 4 R with PEAT_NVFP4, each of these
 * rounded up to 256 bytes; with PEAT_NVFP4 down the columns, there or in
 * peat_quantize_f4, 128 for each column besides.  peat_matmul_f4 and
 * peat_rmsnorm take none, peat_rmsnorm_backward at most 4 bytes for each column and
 * each of two CTAs an SM, and 4 a row of more than 8192 elements (float32: 4096).
 * A gradient list takes 32 bytes for each tensor and 100 KB; one of more than 800
 * takes 40 more for each, and 160 of pinned host memory.
 *
 * The calls can be captured into a CUDA graph, once such a first call has been
 * made (a call that would have to allocate, and a gradient list of more than 800
 * tensors, which the host stages, return PEAT_ERR_UNSUPPORTED).
 * The graph uses the handle's workspace: it lives as long as the handle, and its
 * launches and the handle's calls stay in order on the GPU.
 *
 * The waits inside an 8-bit product of many rows and a 4-bit product are bounded;
 * should one expire, that call's outputs are invalid, and the next product or
 * compare on the handle returns PEAT_ERR_TIMEOUT once.
 */
#ifndef PEAT_OPS_H
#define PEAT_OPS_H

#include "peat.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rounds a matrix x [rows, cols] (PEAT_F32, PEAT_F16 or PEAT_BF16; row r at
 * x + r * ldx elements, ldx >= cols) to 8-bit integers with one scale for
 * each row (axis 0) or each column (axis 1).  Over the row or column,
 *   amax  = max |x|
 *   scale = amax / 127, r = 127 / amax      (float32 divisions)
 *   q     = the nearest integer, ties to even, of the float32 product x * r,
 * so -127 <= q <= 127.  Where r is not finite (amax = 0, or below about
 * 3.7e-37) q = 0 and scale = 0.  A row or column that holds a NaN or an
 * infinity has q = 0 and scale = NaN: every value and every product made
 * from it is NaN.
 *
 * Outputs, each optional (NULL), but for at least one of q and values:
 *   q       axis 0: int8 [rows, cols], row r at q + r * ldq (ldq >= cols);
 *           axis 1: int8 [cols, rows], the transpose, column c at
 *           q + c * ldq (ldq >= rows).  Either way the integers that share a
 *           scale are contiguous, as peat_matmul_i8 reads them.
 *   scale   float32 [rows] (axis 0) or [cols] (axis 1).
 *   values  [rows, cols] of x's type, row r at values + r * ldv (ldv >=
 *           cols): the float32 product q * scale rounded to the type.
 * The outputs must not overlap x.  Fastest with 16-byte aligned rows. */
peat_status_t peat_quantize_i8(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx,
                               peat_dtype_t dtype, int axis, int8_t* q, int64_t ldq, float* scale, void* values,
                               int64_t ldv, peat_stream_t stream);

/* Output types of peat_matmul_i8: PEAT_F32, PEAT_F16, PEAT_BF16, or the
 * integer sums themselves. */
#define PEAT_OUT_I32 100

/* out[m, n] = acc * (a_scale[m] * b_scale[n]) + bias[n], with
 *   acc = sum over k of a[m, k] * b[n, k],
 * the exact integer, rounded once to float32; the scaling and the bias are
 * float32, and the result is rounded once more to a 16-bit out type.
 * a: int8 [M, K], row m at a + m * lda; b: int8 [N, K], row n at b + n * ldb
 * (any int8 value, -128 included; lda, ldb >= K).  a_scale [M], b_scale [N]
 * and bias [N] are float32; a NULL scale is 1, a NULL bias 0.  out: row m at
 * out + m * ldo elements, ldo >= N.  out_dtype PEAT_OUT_I32 stores acc as
 * int32 and takes no scales and no bias.  K <= 131071 (the sums fit 32 bits);
 * K = 0 gives 0 (plus the bias).  out must not overlap the inputs. */
peat_status_t peat_matmul_i8(peat_handle_t h, const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b,
                             int64_t ldb, const float* b_scale, const float* bias, int64_t M, int64_t N, int64_t K,
                             void* out, int64_t ldo, int out_dtype, peat_stream_t stream);

/* An operand of peat_product_i8: a matrix [rows, cols], row r at data + r * ld
 * elements (ld >= cols).  dtype PEAT_INT8: 8-bit integers with their scales
 * (scale: float32 [rows], NULL: 1), axis 0.  dtype PEAT_F32, PEAT_F16 or
 * PEAT_BF16: rounded to such integers as peat_quantize_i8 does, with a scale
 * for each row (axis 0), or for each column (axis 1, whose transpose is then
 * the operand); scale is not read. */
#define PEAT_INT8 101
typedef struct {
  const void* data;
  const float* scale;
  int64_t rows, cols, ld;
  int32_t dtype;
  int32_t axis;
} peat_operand_t;

/* peat_matmul_i8 of two operands that are rounded on the way where they are
 * not integers yet: a's M x K is rows x cols (axis 0) or cols x rows (axis 1),
 * b's N x K likewise, the two K equal.  The results are those of
 * peat_quantize_i8 followed by peat_matmul_i8, in one call and without the
 * integers' detour through the caller.  out_dtype PEAT_F32, PEAT_F16 or
 * PEAT_BF16. */
peat_status_t peat_product_i8(peat_handle_t h, const peat_operand_t* a, const peat_operand_t* b, const float* bias,
                              void* out, int64_t ldo, peat_dtype_t out_dtype, peat_stream_t stream);

/* ---- 4-bit floating point with a scale for each block ----
 *
 * A 4-bit value is +-0, 0.5, 1, 1.5, 2, 3, 4 or 6: one sign bit (bit 3 of its
 * code), two exponent bits, one mantissa bit.  Blocks along the product's axis
 * share a scale:
 *   PEAT_MXFP4  32 values, a power of two 2^e in one byte, e + 127 (255: NaN)
 *   PEAT_NVFP4  16 values, an 8-bit float (4 exponent bits, bias 7, 3 mantissa
 *               bits, sign 0; 0x7f: NaN), below a float32 scale of the whole row
 *               (the row's own, as peat_quantize_i8 has one; elsewhere the format
 *               of this name often has one float32 scale for the whole matrix:
 *               peat_matmul_f4 takes such a matrix with its scale on every row, but
 *               peat_quantize_f4 does not round by a scale that it is given, and by
 *               the rows' scales the blocks' come out otherwise)
 * Codes lie two to a byte, the first in the low half; a row is whole blocks and
 * starts on a 16-byte boundary.  Block scales lie in tiles of 128 rows by 4
 * blocks, 512 bytes: row r of a tile and block k at (r mod 32) * 16 + (r div 32) *
 * 4 + k; the tiles of the first 128 rows come first, in the order of the blocks.
 * A matrix of `rows` rows and `blocks` blocks a row has peat_f4_scale_bytes of
 * them; what lies in the margins of the tiles is zero (or any scale but NaN). */
typedef enum { PEAT_MXFP4 = 0, PEAT_NVFP4 = 1 } peat_f4_t;

/* Bytes of a matrix's block scales: ceil(rows / 128) * ceil(blocks / 4) * 512. */
static inline int64_t peat_f4_scale_bytes(int64_t rows, int64_t blocks) {
  return (rows + 127) / 128 * ((blocks + 3) / 4) * 512;
}

/* Rounds a matrix x [rows, cols] (PEAT_F32, PEAT_F16 or PEAT_BF16; row r at x + r
 * * ldx elements, ldx >= cols) to 4-bit values, with blocks along its rows (axis
 * 0) or down its columns (axis 1).  E2M1(v) is the code nearest to v, ties to the
 * even code, at most 6 in magnitude; all operations are float32 ones.
 *   PEAT_MXFP4  amax = max |x| over the block; e = floor(log2(amax)) - 2, at least
 *               -127 (amax = 0: -127); code = E2M1(x * 2^-e).  A block that holds
 *               a NaN or an infinity has codes 0 and scale NaN.
 *   PEAT_NVFP4  over the row (column): amax = max |x|, scale = amax / 2688, t =
 *               2688 / amax; over the block: b = the 8-bit float nearest to (max
 *               |x| * t) / 6, ties to even; code = E2M1((x * t) * (1 / b)), 0 where
 *               b = 0.  Where t is not finite (amax = 0, or below about 7.9e-36)
 *               scale, b and codes are 0; a row that holds a NaN or an infinity has
 *               b and codes 0 and scale = NaN.
 *
 * Outputs, each optional (NULL), but for at least one of q and values; q needs
 * block_scale, and with PEAT_NVFP4 scale:
 *   q            axis 0: [rows, ceil(cols / block) * block / 2 bytes], row r at q +
 *                r * ldq bytes; axis 1: the transpose, [cols, ceil(rows / block) *
 *                block / 2 bytes].  ldq a multiple of 16; codes beyond the matrix
 *                are 0.
 *   block_scale  peat_f4_scale_bytes(rows of q, blocks of a row), margins 0.
 *   scale        PEAT_NVFP4: float32 [rows] (axis 0) or [cols] (axis 1).
 *   values       [rows, cols] of x's type, row r at values + r * ldv: the code's
 *                value times 2^e, or times b, times scale (each product rounded),
 *                rounded to the type.
 * The outputs must not overlap x; at most 2^30 along the product's axis.  Fastest
 * with 16-byte aligned rows. */
peat_status_t peat_quantize_f4(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx,
                               peat_dtype_t dtype, peat_f4_t format, int axis, uint8_t* q, int64_t ldq,
                               uint8_t* block_scale, float* scale, void* values, int64_t ldv, peat_stream_t stream);

/* out[m, n] = acc * (a_scale[m] * b_scale[n]) + bias[n], with acc the sum over k of
 * the products of the operands' values (codes times block scales), in float32: the
 * values' products are exact, the sum is rounded as it goes, in an order that
 * depends on the sizes and on whether out's rows start on 16-byte boundaries.  Scaling and bias are float32 operations, the result
 * is rounded once more to a 16-bit type.  (A product of two block scales outside
 * float32's range gives infinities, NaN or 0.)
 * a: [M, K], b: [N, K], both of `format`, K whole blocks, rows lda and ldb BYTES
 * apart (multiples of 16).  a_scale [M], b_scale [N] (PEAT_NVFP4 alone) and bias [N]
 * are float32; a NULL scale is 1, a NULL bias 0.  out: row m at out + m * ldo
 * elements, ldo >= N; out_dtype PEAT_F32, PEAT_F16 or PEAT_BF16.  K = 0 gives 0 (plus
 * the bias).  out must not overlap the inputs. */
peat_status_t peat_matmul_f4(peat_handle_t h, peat_f4_t format, const uint8_t* a, int64_t lda,
                             const uint8_t* a_block_scale, const float* a_scale, const uint8_t* b, int64_t ldb,
                             const uint8_t* b_block_scale, const float* b_scale, const float* bias, int64_t M,
                             int64_t N, int64_t K, void* out, int64_t ldo, peat_dtype_t out_dtype,
                             peat_stream_t stream);

/* An operand of peat_product_f4: a matrix [rows, cols].  dtype PEAT_F4: codes with
 * their scales (scale: PEAT_NVFP4 alone, NULL is 1), axis 0, cols whole blocks, rows ld bytes apart.
 * dtype PEAT_F32, PEAT_F16 or PEAT_BF16: rounded as peat_quantize_f4 does, along its
 * rows (axis 0) or columns (axis 1, whose transpose is then the operand), rows ld
 * elements apart; the scales are not read. */
#define PEAT_F4 102
typedef struct {
  const void* data;
  const uint8_t* block_scale;
  const float* scale;
  int64_t rows, cols, ld;
  int32_t dtype;
  int32_t axis;
} peat_operand_f4_t;

/* peat_matmul_f4 of two operands that are rounded on the way where they are not
 * 4-bit values yet: a's M x K is rows x cols (axis 0) or cols x rows (axis 1), b's N
 * x K likewise, the two K equal once they are filled up to whole blocks. */
peat_status_t peat_product_f4(peat_handle_t h, peat_f4_t format, const peat_operand_f4_t* a,
                              const peat_operand_f4_t* b, const float* bias, void* out, int64_t ldo,
                              peat_dtype_t out_dtype, peat_stream_t stream);

/* ---- root-mean-square norm ----
 *
 * The norm that precedes a sublayer's products, of the residual stream with what
 * the sublayer before adds to it, and its output in 8 bits as peat_matmul_i8 takes
 * it.  Over each row of x [rows, cols] (of type dtype), in float32 unless said
 * otherwise,
 *   s     = x + residual, rounded to dtype (no residual: x)
 *   v     = (sum of s^2) / cols, summed in twice the precision, rounded once
 *   rstd  = 1 / sqrt(v + eps)
 *   y     = (s * rstd) * weight
 *   scale = amax / 127 and q = the nearest integer of y * (127 / amax), amax = max
 *           |y|, with all of peat_quantize_i8's rules (float32 y, not the rounded).
 * weight [cols] is of type dtype or PEAT_F32.  A NaN or an infinity in a row goes
 * where the formulas take it; no square overflows or underflows.  Rows of no columns
 * have scale 0 and rstd NaN (0 / 0).
 * Outputs, each optional (NULL), one at least: sum (s), y and values (q * scale)
 * [rows, cols] of type dtype, q int8 [rows, cols], scale and rstd float32 [rows].
 * sum may be x or residual itself (the same rows at the same distance); else no
 * output overlaps an input or another output. */
peat_status_t peat_rmsnorm(peat_handle_t h, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                           const void* weight, peat_dtype_t weight_dtype, int64_t rows, int64_t cols,
                           peat_dtype_t dtype, float eps, void* sum, int64_t lds, void* y, int64_t ldy, int8_t* q,
                           int64_t ldq, float* scale, void* values, int64_t ldv, float* rstd, peat_stream_t stream);

/* The norm's gradients, of grad = dL/dy and, where the stream goes on beside the
 * sublayer, grad_sum = dL/ds (NULL: none), from x = s (peat_rmsnorm's sum) and its
 * rstd.  With n = x * rstd, g = grad * weight, c = (sum of g * n) / cols,
 *   grad_x      = rstd * (g - n * c) + grad_sum, rounded to dtype: the gradient of
 *                 x and of the residual alike (float32 operations, n * c and its
 *                 subtraction one of them)
 *   grad_weight = the sum over the rows of grad * n, float32 [cols].
 * (Rounding to 8 bits passes gradients through: grad is then that of values.)  Sums
 * are float32, in an order that depends on the sizes and on whether all rows, and the
 * weight, are whole 16-byte units on 16-byte boundaries.  Each output may be
 * NULL, not both; no rows give grad_weight 0.  cols <= 2^27.  grad_x may be grad or
 * grad_sum itself (the same rows at the same distance), else no output overlaps an
 * input. */
peat_status_t peat_rmsnorm_backward(peat_handle_t h, const void* grad, int64_t ldg, const void* grad_sum,
                                    int64_t ldr, const void* x, int64_t ldx, const void* weight,
                                    peat_dtype_t weight_dtype, const float* rstd, int64_t rows, int64_t cols,
                                    peat_dtype_t dtype, void* grad_x, int64_t ldo, float* grad_weight,
                                    peat_stream_t stream);

/* One tensor of a gradient list (a HOST array, copied before the call
 * returns): n contiguous elements of type dtype (PEAT_F32, PEAT_F16,
 * PEAT_BF16) at g.  out is peat_grad_clip's output: g itself (in place) or
 * another buffer that overlaps none of the list's tensors; peat_grad_norm
 * ignores it.  n = 0 is allowed (the pointers are not read). */
typedef struct {
  const void* g;
  void* out;
  int64_t n;
  int32_t dtype;
  int32_t reserved; /* 0 */
} peat_grad_t;

/* What a norm or clipping call found (device memory, 16 bytes). */
typedef struct {
  float norm;          /* over all tensors */
  float coef;          /* peat_grad_clip: the clipping factor c; peat_grad_norm: 1 */
  uint64_t n_bad;      /* elements that are NaN or infinite */
} peat_gradnorm_t;

typedef enum {
  PEAT_NORM_2 = 0,   /* sqrt(sum x^2) */
  PEAT_NORM_1 = 1,   /* sum |x| */
  PEAT_NORM_INF = 2  /* max |x| */
} peat_norm_t;

/* What peat_grad_clip does where some element is NaN or infinite. */
typedef enum {
  PEAT_BAD_PROPAGATE = 0, /* nothing special: c follows from the norm (NaN, or 0 for an infinite norm) */
  PEAT_BAD_ZERO = 1,      /* c = 0 and every output is +0: the step changes nothing */
  PEAT_BAD_KEEP = 2       /* c = 1: the gradients come out scaled by unscale alone */
} peat_bad_t;

/* Norm of x = unscale * g over all tensors of the list, and of each tensor
 * (norms: float32 [count] or NULL).  unscale (finite, > 0) undoes a loss
 * scale.  Squares are summed in float32 over at most 64 elements and beyond
 * that with a compensation, in a fixed order: the same list gives the same
 * bits on every call.  Neither squares nor sums overflow or underflow at any
 * magnitude of g.  An infinite element makes its tensor's norm and the whole
 * norm +inf, a NaN makes them NaN.  An empty list has norm 0. */
peat_status_t peat_grad_norm(peat_handle_t h, const peat_grad_t* list, int64_t count, peat_norm_t type,
                             float unscale, peat_gradnorm_t* result, float* norms, peat_stream_t stream);

/* The same, and every tensor scaled: out = g * (unscale * c), one float32
 * product of each element, rounded once to its type, with
 *   c = min(1, max_norm / (norm + eps))     (float32; NaN stays NaN)
 * max_norm >= 0 (may be +inf), eps >= 0.  With unscale * c = 1 an in-place
 * tensor is not touched (its values would not change). */
peat_status_t peat_grad_clip(peat_handle_t h, const peat_grad_t* list, int64_t count, peat_norm_t type,
                             float unscale, float max_norm, float eps, peat_bad_t bad, peat_gradnorm_t* result,
                             float* norms, peat_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif
