/*
 * peat_ops.h -- the operators of libpeat that a playback step runs beside the
 * compare: a linear layer's products in 8-bit integers, and the norm and the
 * clipping of a list of gradients.
 *
 * Playback FI (Alg. 1) computes a layer's forward output, its input gradient
 * and its weight gradient again at a lower precision from the recorded
 * (activation, weight, output gradient), and scores them against the golden
 * ones.  Here the lower precision is 8-bit integers with one scale for each
 * row of either operand: peat_quantize_i8 makes the operands,
 * peat_matmul_i8 multiplies them, peat_product_i8 does both.  A training step
 * ends with the norm over all its gradient tensors, by which they are clipped:
 * peat_grad_norm and peat_grad_clip.
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
 * taken; operands that peat_product_i8 rounds add a byte for each element.  A
 * gradient list takes 32 bytes for each tensor and 100 KB; one of more than 800
 * takes 40 more for each, and 160 of pinned host memory.
 *
 * The calls can be captured into a CUDA graph, once such a first call has been
 * made (a call that would have to allocate, and a gradient list of more than 800
 * tensors, which the host stages, return PEAT_ERR_UNSUPPORTED).
 * The graph uses the handle's workspace: it lives as long as the handle, and its
 * launches and the handle's calls stay in order on the GPU.
 *
 * The waits inside a product of many rows are bounded; should one expire, that
 * call's outputs are invalid, and the next product or compare on the handle
 * returns PEAT_ERR_TIMEOUT once.
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
