// Host side of the 4-bit products and the root-mean-square norm declared in
// include/peat_ops.h: argument checks, workspace, launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "ops_state.h"

namespace {

using peat::aligned;
using peat::cuda_fail;
using peat::DeviceGuard;
using peat::fail;
using peat::guarded;
using peat::OpsState;
using peat::type_bytes;

// (rows are counted in 32 bits with their margins)
constexpr int64_t MAX_ROWS = peat::MAX_DIM - 255;
constexpr int64_t MAX_K = (int64_t)1 << 30;

int64_t block_of(int format) { return format == PEAT_MXFP4 ? 32 : 16; }
int64_t blocks_of(int format, int64_t k) { return (k + block_of(format) - 1) / block_of(format); }
int64_t tiles_of(int format, int64_t k) { return (blocks_of(format, k) + 3) / 4; }
bool format_ok(int format) { return format == PEAT_MXFP4 || format == PEAT_NVFP4; }

// the checks of a quantisation, and its launch's parameters but for the workspace
peat_status_t quant_params(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int format,
                           int axis, uint8_t* q, int64_t ldq, uint8_t* block_scale, float* scale, void* values, int64_t ldv,
                           peat::Quant4Params* p) {
  const int B = type_bytes(dtype);
  if (!B) return fail(h, PEAT_ERR_INVALID_ARG, "dtype must be PEAT_F32, PEAT_F16 or PEAT_BF16");
  if (!format_ok(format)) return fail(h, PEAT_ERR_INVALID_ARG, "format must be PEAT_MXFP4 or PEAT_NVFP4");
  if (axis != 0 && axis != 1) return fail(h, PEAT_ERR_INVALID_ARG, "axis must be 0 (rows) or 1 (columns)");
  if (rows < 0 || cols < 0) return fail(h, PEAT_ERR_INVALID_ARG, "rows or cols < 0");
  if (rows > MAX_ROWS || cols > MAX_ROWS) return fail(h, PEAT_ERR_UNSUPPORTED, "rows or cols above 2^31 - 256");
  if (ldx < cols) return fail(h, PEAT_ERR_INVALID_ARG, "ldx < cols");
  if (format == PEAT_MXFP4 && scale) return fail(h, PEAT_ERR_INVALID_ARG, "PEAT_MXFP4 has no float32 scales");
  const int64_t k = axis ? rows : cols, width = blocks_of(format, k) * block_of(format);
  if (k > MAX_K) return fail(h, PEAT_ERR_UNSUPPORTED, "more than 2^30 along the product's axis");
  if (q && (ldq < width / 2 || (ldq % 16 && (axis ? cols : rows) > 1) || !aligned(q, 16)))
    return fail(h, PEAT_ERR_INVALID_ARG, "q's rows must hold whole blocks and start on 16-byte boundaries");
  if (block_scale && !aligned(block_scale, 16)) return fail(h, PEAT_ERR_INVALID_ARG, "block_scale must be 16-byte aligned");
  if (values && ldv < cols) return fail(h, PEAT_ERR_INVALID_ARG, "ldv < cols");
  if (rows > 0 && cols > 0) {
    if (!x) return fail(h, PEAT_ERR_INVALID_ARG, "x is NULL");
    if (!q && !values) return fail(h, PEAT_ERR_INVALID_ARG, "q and values are both NULL");
    if (q && !block_scale) return fail(h, PEAT_ERR_INVALID_ARG, "q without block_scale");
    if (q && format == PEAT_NVFP4 && !scale) return fail(h, PEAT_ERR_INVALID_ARG, "q without scale: PEAT_NVFP4 needs the rows' scales");
    if (!aligned(x, B)) return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  }
  if ((values && !aligned(values, B)) || (scale && !aligned(scale, 4)))
    return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  const int E = 16 / B;
  std::memset(p, 0, sizeof(*p));
  p->x = x;
  p->rows = rows;
  p->cols = cols;
  p->ldx = ldx;
  p->q = q;
  p->ldq = ldq;
  p->width = width;
  p->block_scale = block_scale;
  p->tiles = tiles_of(format, k);
  p->scale = scale;
  p->values = values;
  p->ldv = ldv;
  p->vec_x = aligned(x, 16) && (ldx % E == 0 || rows <= 1);
  p->vec_v = values && aligned(values, 16) && (ldv % E == 0 || rows <= 1);
  p->pairs = aligned(x, 2 * B) && (ldx % 2 == 0 || rows <= 1);
  p->pairs_v = aligned(values, 2 * B) && (ldv % 2 == 0 || rows <= 1);
  return PEAT_OK;
}

peat_status_t round4(peat_handle_t h, int dtype, int format, int axis, peat::Quant4Params* p, cudaStream_t st) {
  cudaError_t e = peat::launch_quant4(dtype, format, axis, *p, h->nsm, st);
  return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "4-bit quantisation launch");
}
// the columns' maxima over parts of the rows, which nvfp4 by column needs
size_t tops_bytes(int format, int axis, int64_t cols) {
  return axis && format == PEAT_NVFP4 ? sizeof(unsigned int) * (size_t)peat::QUANT4_CHUNKS * (size_t)cols : 0;
}

peat_status_t quantize(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int format, int axis,
                       uint8_t* q, int64_t ldq, uint8_t* block_scale, float* scale, void* values, int64_t ldv, cudaStream_t st) {
  peat::Quant4Params p;
  peat_status_t ps = quant_params(h, x, rows, cols, ldx, dtype, format, axis, q, ldq, block_scale, scale, values, ldv, &p);
  if (ps != PEAT_OK) return ps;
  const int64_t across = axis ? cols : rows;
  if (across == 0 || (p.tiles == 0 && !scale)) return PEAT_OK;
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  if (p.tiles == 0) {  // rows of nothing
    cudaError_t e = cudaMemsetAsync(scale, 0, sizeof(float) * (size_t)across, st);
    return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "cudaMemsetAsync(scale)");
  }
  if (const size_t need = tops_bytes(format, axis, cols)) {
    OpsState* s = nullptr;
    ps = peat::ops_state(h, st, &s);
    if (ps == PEAT_OK) ps = peat::grow(h, &s->tops, &s->tops_cap, need);
    if (ps != PEAT_OK) return ps;
    p.tops = static_cast<unsigned int*>(s->tops);
  }
  return round4(h, dtype, format, axis, &p, st);
}

// checks of a product's output and sizes
peat_status_t product_ok(peat_handle_t h, const float* sa, const float* sb, const float* bias, int64_t M, int64_t N,
                         int64_t K, const void* out, int64_t ldo, int out_dtype) {
  const int B = type_bytes(out_dtype);
  if (!B) return fail(h, PEAT_ERR_INVALID_ARG, "out_dtype must be PEAT_F32, PEAT_F16 or PEAT_BF16");
  if (ldo < N) return fail(h, PEAT_ERR_INVALID_ARG, "ldo is less than a row");
  if (M > MAX_ROWS || N > MAX_ROWS || K > MAX_K)
    return fail(h, PEAT_ERR_UNSUPPORTED, "M or N above 2^31 - 256, or K above 2^30");
  if (M == 0 || N == 0) return PEAT_OK;
  // tiles are counted in 32 bits
  if (((M + 127) / 128) * ((N + 127) / 128) > ((int64_t)1 << 27))
    return fail(h, PEAT_ERR_UNSUPPORTED, "the output is too large for one call");
  if (!out) return fail(h, PEAT_ERR_INVALID_ARG, "out is NULL");
  if (!aligned(out, B) || (sa && !aligned(sa, 4)) || (sb && !aligned(sb, 4)) || (bias && !aligned(bias, 4)))
    return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  return peat::expired(h);
}
peat_status_t operand_ok(peat_handle_t h, const uint8_t* q, int64_t ld, const uint8_t* block_scale, int64_t rows) {
  if (!q || !block_scale) return fail(h, PEAT_ERR_INVALID_ARG, "an operand's codes or block scales are NULL");
  if (!aligned(q, 16) || (rows > 1 && ld % 16) || !aligned(block_scale, 16))
    return fail(h, PEAT_ERR_INVALID_ARG, "an operand's rows and block scales must start on 16-byte boundaries");
  if (ld > ((int64_t)1 << 39)) return fail(h, PEAT_ERR_UNSUPPORTED, "rows more than 2^39 bytes apart");
  return PEAT_OK;
}
peat_status_t multiply(peat_handle_t h, int format, const peat::Mm4Params& p, int out_dtype, cudaStream_t st) {
  cudaError_t e = peat::launch_mm4(format, out_dtype, p, h->status_dev, peat::wait_limit(h), h->nsm, st);
  return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "4-bit product launch");
}

peat_status_t matmul(peat_handle_t h, int format, const uint8_t* a, int64_t lda, const uint8_t* abs, const float* sa,
                     const uint8_t* b, int64_t ldb, const uint8_t* bbs, const float* sb, const float* bias, int64_t M, int64_t N,
                     int64_t K, void* out, int64_t ldo, int out_dtype, cudaStream_t st) {
  if (!format_ok(format)) return fail(h, PEAT_ERR_INVALID_ARG, "format must be PEAT_MXFP4 or PEAT_NVFP4");
  if (M < 0 || N < 0 || K < 0) return fail(h, PEAT_ERR_INVALID_ARG, "M, N or K < 0");
  if (format == PEAT_MXFP4 && (sa || sb)) return fail(h, PEAT_ERR_INVALID_ARG, "PEAT_MXFP4 has no float32 scales");
  if (K % block_of(format)) return fail(h, PEAT_ERR_INVALID_ARG, "K must be whole blocks (the quantiser fills a row's last one with zeros)");
  if (lda < K / 2 || ldb < K / 2) return fail(h, PEAT_ERR_INVALID_ARG, "lda or ldb is less than a row");
  peat_status_t ps = product_ok(h, sa, sb, bias, M, N, K, out, ldo, out_dtype);
  if (ps != PEAT_OK || M == 0 || N == 0) return ps;
  if (K > 0) ps = operand_ok(h, a, lda, abs, M);
  if (K > 0 && ps == PEAT_OK) ps = operand_ok(h, b, ldb, bbs, N);
  if (ps != PEAT_OK) return ps;
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  if (K == 0) sa = sb = nullptr;  // (nothing to scale, and 0 x NaN must not get through)
  return multiply(h, format, peat::Mm4Params{a, b, lda, ldb, abs, bbs, sa, sb, bias, out, ldo, M, N, K}, out_dtype, st);
}

// An operand as the product takes it: as it is, or its place in the workspace at
// *at, which moves on (ws NULL: only counted).
struct Operand {
  const uint8_t* q;
  const uint8_t* block_scale;
  const float* scale;
  int64_t rows, K, ld;
};
size_t up(size_t n) { return (n + 255) / 256 * 256; }
bool valid(const peat_operand_f4_t* o, int format) {
  if (!o || o->rows < 0 || o->cols < 0 || o->ld < 0 || o->rows > MAX_ROWS || o->cols > MAX_ROWS) return false;
  if (o->dtype == PEAT_F4) return o->axis == 0 && o->cols % block_of(format) == 0 && o->ld >= o->cols / 2;
  return type_bytes(o->dtype) != 0 && (o->axis == 0 || o->axis == 1) && o->ld >= o->cols;
}
Operand operand_of(const peat_operand_f4_t& o, int format, char* ws, size_t* at) {
  Operand r;
  r.rows = o.axis ? o.cols : o.rows;
  const int64_t k = o.axis ? o.rows : o.cols;
  r.K = blocks_of(format, k) * block_of(format);
  if (o.dtype == PEAT_F4) {
    r.q = static_cast<const uint8_t*>(o.data);
    r.block_scale = o.block_scale;
    r.scale = o.scale;
    r.ld = o.ld;
    return r;
  }
  r.ld = (r.K / 2 + 15) / 16 * 16;
  r.scale = format == PEAT_NVFP4 ? reinterpret_cast<const float*>(ws + *at) : nullptr;
  if (format == PEAT_NVFP4) *at += up((size_t)r.rows * sizeof(float));
  r.block_scale = reinterpret_cast<const uint8_t*>(ws + *at);
  *at += up((size_t)((r.rows + 127) / 128) * (size_t)tiles_of(format, k) * 512);
  r.q = reinterpret_cast<const uint8_t*>(ws + *at);
  *at += up((size_t)r.rows * (size_t)r.ld);
  return r;
}

peat_status_t product(peat_handle_t h, int format, const peat_operand_f4_t* a, const peat_operand_f4_t* b, const float* bias,
                      void* out, int64_t ldo, int out_dtype, cudaStream_t st) {
  if (!format_ok(format)) return fail(h, PEAT_ERR_INVALID_ARG, "format must be PEAT_MXFP4 or PEAT_NVFP4");
  if (!valid(a, format) || !valid(b, format))
    return fail(h, PEAT_ERR_INVALID_ARG, "an operand is NULL, or its sizes, dtype or axis are not valid");
  const peat_operand_f4_t* in[2] = {a, b};
  for (int i = 0; i < 2; i++)
    if (format == PEAT_MXFP4 && in[i]->dtype == PEAT_F4 && in[i]->scale)
      return fail(h, PEAT_ERR_INVALID_ARG, "PEAT_MXFP4 has no float32 scales");
  size_t need = 0;
  Operand op[2] = {operand_of(*a, format, nullptr, &need), operand_of(*b, format, nullptr, &need)};
  if (op[0].K != op[1].K) return fail(h, PEAT_ERR_INVALID_ARG, "the operands differ in K");
  const int64_t M = op[0].rows, N = op[1].rows, K = op[0].K;
  peat_status_t ps = product_ok(h, a->dtype == PEAT_F4 ? a->scale : nullptr, b->dtype == PEAT_F4 ? b->scale : nullptr, bias,
                                M, N, K, out, ldo, out_dtype);
  if (ps != PEAT_OK || M == 0 || N == 0) return ps;
  for (int i = 0; i < 2 && K > 0; i++) {
    if (!in[i]->data) return fail(h, PEAT_ERR_INVALID_ARG, "an operand's data is NULL");
    if (in[i]->dtype == PEAT_F4) ps = operand_ok(h, op[i].q, op[i].ld, op[i].block_scale, op[i].rows);
    if (ps != PEAT_OK) return ps;
  }
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  OpsState* s = nullptr;
  ps = peat::ops_state(h, st, &s);
  if (ps == PEAT_OK) ps = peat::grow(h, &s->rounded, &s->rounded_cap, need);
  // (each operand's maxima have a place of their own: the second is rounded beside the first)
  size_t tops[2] = {0, 0};
  for (int i = 0; i < 2; i++)
    if (in[i]->dtype != PEAT_F4) tops[i] = tops_bytes(format, in[i]->axis, in[i]->cols);
  if (ps == PEAT_OK && tops[0] + tops[1]) ps = peat::grow(h, &s->tops, &s->tops_cap, tops[0] + tops[1]);
  if (ps != PEAT_OK) return ps;
  size_t at = 0;
  bool beside = false;
  for (int i = 0; i < 2; i++) {
    op[i] = operand_of(*in[i], format, static_cast<char*>(s->rounded), &at);
    if (in[i]->dtype == PEAT_F4 || K == 0) continue;
    peat::Quant4Params q;
    ps = quant_params(h, in[i]->data, in[i]->rows, in[i]->cols, in[i]->ld, in[i]->dtype, format, in[i]->axis,
                      const_cast<uint8_t*>(op[i].q), op[i].ld, const_cast<uint8_t*>(op[i].block_scale),
                      const_cast<float*>(op[i].scale), nullptr, 0, &q);
    q.tops = reinterpret_cast<unsigned int*>(static_cast<char*>(s->tops) + (i ? tops[0] : 0));
    q.overlap = beside;
    beside = true;
    if (ps == PEAT_OK) ps = round4(h, in[i]->dtype, format, in[i]->axis, &q, st);
    if (ps != PEAT_OK) return ps;
  }
  // (without k there is nothing to scale)
  const float *sa = K ? op[0].scale : nullptr, *sb = K ? op[1].scale : nullptr;
  return multiply(h, format, peat::Mm4Params{op[0].q, op[1].q, op[0].ld, op[1].ld, op[0].block_scale, op[1].block_scale, sa, sb, bias,
                                             out, ldo, M, N, K}, out_dtype, st);
}

// ---- root-mean-square norm ----
bool vec(const void* p, int64_t ld, int64_t rows, int bytes) {
  return aligned(p, 16) && (ld * bytes % 16 == 0 || rows <= 1);
}
peat_status_t norm_sizes(peat_handle_t h, int64_t rows, int64_t cols, int dtype, int weight_dtype) {
  if (!type_bytes(dtype)) return fail(h, PEAT_ERR_INVALID_ARG, "dtype must be PEAT_F32, PEAT_F16 or PEAT_BF16");
  if (weight_dtype != PEAT_F32 && weight_dtype != dtype)
    return fail(h, PEAT_ERR_INVALID_ARG, "weight_dtype must be dtype or PEAT_F32");
  if (rows < 0 || cols < 0) return fail(h, PEAT_ERR_INVALID_ARG, "rows or cols < 0");
  if (rows > MAX_ROWS || cols > MAX_ROWS) return fail(h, PEAT_ERR_UNSUPPORTED, "rows or cols above 2^31 - 256");
  return PEAT_OK;
}

peat_status_t rmsnorm(peat_handle_t h, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                      int weight_dtype, int64_t rows, int64_t cols, int dtype, float eps, void* sum, int64_t lds, void* y,
                      int64_t ldy, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv, float* rstd, cudaStream_t st) {
  peat_status_t ps = norm_sizes(h, rows, cols, dtype, weight_dtype);
  if (ps != PEAT_OK) return ps;
  const int B = type_bytes(dtype), E = 16 / B;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(h, PEAT_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (ldx < cols || (residual && ldr < cols) || (sum && lds < cols) || (y && ldy < cols) || (q && ldq < cols) || (values && ldv < cols))
    return fail(h, PEAT_ERR_INVALID_ARG, "a matrix's row distance is less than a row");
  if (rows == 0) return PEAT_OK;
  if (cols > 0 && (!x || !weight)) return fail(h, PEAT_ERR_INVALID_ARG, "x or weight is NULL");
  if (cols > 0 && !sum && !y && !q && !scale && !values && !rstd) return fail(h, PEAT_ERR_INVALID_ARG, "no output is asked for");
  for (const void* p : {x, residual, (const void*)sum, (const void*)y, (const void*)values})
    if (!aligned(p, B)) return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  if (!aligned(weight, type_bytes(weight_dtype)) || !aligned(scale, 4) || !aligned(rstd, 4))
    return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  if (cols == 0) {  // rows of nothing: bytes of zeros, and of a NaN
    cudaError_t e = scale ? cudaMemsetAsync(scale, 0, sizeof(float) * (size_t)rows, st) : cudaSuccess;
    if (e == cudaSuccess && rstd) e = cudaMemsetAsync(rstd, 0xff, sizeof(float) * (size_t)rows, st);
    return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "cudaMemsetAsync(scale, rstd)");
  }
  peat::RmsParams p;
  p.x = x;
  p.ldx = ldx;
  p.residual = residual;
  p.ldr = ldr;
  p.weight = weight;
  p.weight_f32 = weight_dtype == PEAT_F32;
  p.rows = rows;
  p.cols = cols;
  p.eps = eps;
  p.sum = sum;
  p.lds = lds;
  p.y = y;
  p.ldy = ldy;
  p.q = q;
  p.ldq = ldq;
  p.scale = scale;
  p.values = values;
  p.ldv = ldv;
  p.rstd = rstd;
  p.grid = cols % E == 0 && aligned(weight, 16) && vec(x, ldx, rows, B) && (!residual || vec(residual, ldr, rows, B)) &&
           (!sum || vec(sum, lds, rows, B)) && (!y || vec(y, ldy, rows, B)) && (!values || vec(values, ldv, rows, B)) &&
           (!q || (aligned(q, E) && (ldq % E == 0 || rows <= 1)));
  cudaError_t e = peat::launch_rmsnorm(dtype, p, h->nsm, st);
  return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "norm launch");
}

peat_status_t rmsnorm_backward(peat_handle_t h, const void* grad, int64_t ldg, const void* grad_sum, int64_t ldr, const void* x,
                               int64_t ldx, const void* weight, int weight_dtype, const float* rstd, int64_t rows, int64_t cols,
                               int dtype, void* grad_x, int64_t ldo, float* grad_weight, cudaStream_t st) {
  peat_status_t ps = norm_sizes(h, rows, cols, dtype, weight_dtype);
  if (ps != PEAT_OK) return ps;
  const int B = type_bytes(dtype);
  if (ldg < cols || ldx < cols || (grad_sum && ldr < cols) || (grad_x && ldo < cols))
    return fail(h, PEAT_ERR_INVALID_ARG, "a matrix's row distance is less than a row");
  if (cols > ((int64_t)1 << 27)) return fail(h, PEAT_ERR_UNSUPPORTED, "cols above 2^27");
  if (cols == 0) return PEAT_OK;
  if (rows > 0 && (!grad || !x || !weight || !rstd)) return fail(h, PEAT_ERR_INVALID_ARG, "grad, x, weight or rstd is NULL");
  if (rows > 0 && !grad_x && !grad_weight) return fail(h, PEAT_ERR_INVALID_ARG, "grad_x and grad_weight are both NULL");
  for (const void* p : {grad, grad_sum, x, (const void*)grad_x})
    if (!aligned(p, B)) return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  if (!aligned(weight, type_bytes(weight_dtype)) || !aligned(rstd, 4) || !aligned(grad_weight, 4))
    return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  if (rows == 0 && !grad_weight) return PEAT_OK;
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  OpsState* s = nullptr;
  const peat::RmsBackPlan plan = peat::rms_back_plan(dtype, rows, cols, h->nsm);
  const size_t parts = grad_weight ? sizeof(float) * (size_t)plan.ctas * (size_t)cols : 0, at = (parts + 255) / 256 * 256;
  const size_t need = at + (plan.longer ? sizeof(float) * (size_t)rows : 0);
  ps = peat::ops_state(h, st, &s);
  if (ps == PEAT_OK) ps = peat::grow(h, &s->norm, &s->norm_cap, need);
  if (ps != PEAT_OK) return ps;
  peat::RmsBackParams p;
  std::memset(&p, 0, sizeof(p));
  p.grad = grad;
  p.ldg = ldg;
  p.stream = grad_sum;
  p.ldr = ldr;
  p.x = x;
  p.ldx = ldx;
  p.weight = weight;
  p.weight_f32 = weight_dtype == PEAT_F32;
  p.rstd = rstd;
  p.rows = rows;
  p.cols = cols;
  p.grad_x = grad_x;
  p.ldo = ldo;
  p.grad_weight = grad_weight;
  p.parts = static_cast<float*>(s->norm);
  p.dots = reinterpret_cast<float*>(static_cast<char*>(s->norm) + at);
  p.grid = cols % (16 / B) == 0 && aligned(weight, 16) && vec(grad, ldg, rows, B) && vec(x, ldx, rows, B) &&
           (!grad_sum || vec(grad_sum, ldr, rows, B)) && (!grad_x || vec(grad_x, ldo, rows, B));
  cudaError_t e = peat::launch_rmsnorm_backward(dtype, plan, p, st);
  return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "norm gradient launch");
}

}  // namespace

extern "C" {

peat_status_t peat_quantize_f4(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx, peat_dtype_t dtype,
                               peat_f4_t format, int axis, uint8_t* q, int64_t ldq, uint8_t* block_scale, float* scale,
                               void* values, int64_t ldv, peat_stream_t stream) {
  return guarded(h, [&] {
    return quantize(h, x, rows, cols, ldx, dtype, format, axis, q, ldq, block_scale, scale, values, ldv,
                    reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_matmul_f4(peat_handle_t h, peat_f4_t format, const uint8_t* a, int64_t lda, const uint8_t* a_block_scale,
                             const float* a_scale, const uint8_t* b, int64_t ldb, const uint8_t* b_block_scale,
                             const float* b_scale, const float* bias, int64_t M, int64_t N, int64_t K, void* out, int64_t ldo,
                             peat_dtype_t out_dtype, peat_stream_t stream) {
  return guarded(h, [&] {
    return matmul(h, format, a, lda, a_block_scale, a_scale, b, ldb, b_block_scale, b_scale, bias, M, N, K, out, ldo, out_dtype,
                  reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_product_f4(peat_handle_t h, peat_f4_t format, const peat_operand_f4_t* a, const peat_operand_f4_t* b,
                              const float* bias, void* out, int64_t ldo, peat_dtype_t out_dtype, peat_stream_t stream) {
  return guarded(h, [&] { return product(h, format, a, b, bias, out, ldo, out_dtype, reinterpret_cast<cudaStream_t>(stream)); });
}

peat_status_t peat_rmsnorm(peat_handle_t h, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                           peat_dtype_t weight_dtype, int64_t rows, int64_t cols, peat_dtype_t dtype, float eps, void* sum,
                           int64_t lds, void* y, int64_t ldy, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                           float* rstd, peat_stream_t stream) {
  return guarded(h, [&] {
    return rmsnorm(h, x, ldx, residual, ldr, weight, weight_dtype, rows, cols, dtype, eps, sum, lds, y, ldy, q, ldq, scale, values,
                   ldv, rstd, reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_rmsnorm_backward(peat_handle_t h, const void* grad, int64_t ldg, const void* grad_sum, int64_t ldr,
                                    const void* x, int64_t ldx, const void* weight, peat_dtype_t weight_dtype, const float* rstd,
                                    int64_t rows, int64_t cols, peat_dtype_t dtype, void* grad_x, int64_t ldo,
                                    float* grad_weight, peat_stream_t stream) {
  return guarded(h, [&] {
    return rmsnorm_backward(h, grad, ldg, grad_sum, ldr, x, ldx, weight, weight_dtype, rstd, rows, cols, dtype, grad_x, ldo,
                            grad_weight, reinterpret_cast<cudaStream_t>(stream));
  });
}

}  // extern "C"
