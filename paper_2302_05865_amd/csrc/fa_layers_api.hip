// C ABI of the workers' backward pass (see include/fa.h): argument checking and the order in which the kernels are
// enqueued.  No state, no allocation, nothing copied: a call is kernel launches alone.
#include <hip/hip_runtime.h>

#include <math.h>

#include "fa.h"
#include "fa_layers.h"

namespace {

bool known(int dtype) { return dtype == FA_F32 || dtype == FA_BF16; }
int bytes_of(int dtype) { return dtype == FA_F32 ? 4 : 2; }

// a matrix of `rows` rows of `width` elements, `ld` apart; any place that its element type may have
bool matrix(const void* x, int64_t ld, int64_t rows, int64_t width, int dtype) {
  if (rows == 0) return true;
  if (!x || ((uintptr_t)x & (uintptr_t)(bytes_of(dtype) - 1)) != 0) return false;
  return rows == 1 || (ld >= width && ld <= INT64_MAX / 4 / rows);
}
bool params(const void* x, int dtype) { return !x || ((uintptr_t)x & (uintptr_t)(bytes_of(dtype) - 1)) == 0; }
bool floats(const float* x) { return !x || ((uintptr_t)x & 3u) == 0; }
bool checkpoint(const int8_t* codes, const uint8_t* exponents, int64_t rows) {
  return rows == 0 || (codes && exponents && ((uintptr_t)codes & 15u) == 0 && ((uintptr_t)exponents & 3u) == 0);
}
bool extent(int64_t rows, int features, int most) {
  return rows >= 0 && rows <= FA_ROWS_MAX && features >= 1 && features <= most;
}
// the workers' rows one after the other, from their numbers; false: a negative one, or they add up to too many
bool row_blocks(const int64_t* sizes, int p, fa_row_blocks* b) {
  if (!sizes || p < 1 || p > FA_P_MAX) return false;
  b->p = p;
  b->row0[0] = 0;
  for (int w = 0; w < FA_P_MAX; ++w) {
    if (w < p && (sizes[w] < 0 || sizes[w] > FA_ROWS_MAX - b->row0[w])) return false;
    b->row0[w + 1] = b->row0[w] + (w < p ? sizes[w] : 0);
  }
  return true;
}

}  // namespace

extern "C" int64_t fa_checkpoint_code_pitch(int features) { return features < 1 ? 0 : fa_code_pitch(features); }
extern "C" int64_t fa_checkpoint_exponent_pitch(int features) { return features < 1 ? 0 : fa_exponent_pitch(features); }

extern "C" fa_status fa_checkpoint_pack(const void* x, int64_t ldx, int64_t rows, int features, int dtype, int8_t* codes,
                                        uint8_t* exponents, void* stream) {
  if (!known(dtype) || !extent(rows, features, FA_FEATURES_MAX) || !matrix(x, ldx, rows, features, dtype) ||
      !checkpoint(codes, exponents, rows))
    return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  return fa_launch_checkpoint_pack(x, ldx, rows, features, dtype, codes, exponents, (hipStream_t)stream) == hipSuccess
             ? FA_OK : FA_ERR_DEVICE;
}

extern "C" fa_status fa_checkpoint_unpack(const int8_t* codes, const uint8_t* exponents, int64_t rows, int features, int dtype,
                                          void* x, int64_t ldx, void* stream) {
  if (!known(dtype) || !extent(rows, features, FA_FEATURES_MAX) || !matrix(x, ldx, rows, features, dtype) ||
      !checkpoint(codes, exponents, rows))
    return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  return fa_launch_checkpoint_unpack(codes, exponents, rows, features, dtype, x, ldx, (hipStream_t)stream) == hipSuccess
             ? FA_OK : FA_ERR_DEVICE;
}

extern "C" fa_status fa_layer_norm(const void* x, int64_t ldx, int64_t rows, int features, int dtype, const void* gamma,
                                   const void* beta, int param_dtype, double eps, void* y, int64_t ldy, float* mean,
                                   float* rstd, int8_t* codes, uint8_t* exponents, void* stream) {
  if (!known(dtype) || !known(param_dtype) || !extent(rows, features, FA_NORM_FEATURES_MAX) ||
      !matrix(x, ldx, rows, features, dtype) || !matrix(y, ldy, rows, features, dtype) || (rows > 0 && x == y) ||
      !params(gamma, param_dtype) || !params(beta, param_dtype) || !floats(mean) || !floats(rstd) || !(eps >= 0.0) ||
      !isfinite(eps) || (codes == nullptr) != (exponents == nullptr) || (codes && !checkpoint(codes, exponents, rows)))
    return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  fa_norm_args a;
  a.x = x; a.gamma = gamma; a.beta = beta; a.y = y;
  a.mean = mean; a.rstd = rstd; a.codes = codes; a.exponents = exponents;
  a.ldx = ldx; a.ldy = ldy; a.rows = rows;
  a.features = features; a.param_bf16 = param_dtype == FA_BF16; a.eps = (float)eps;
  return fa_launch_layer_norm(a, dtype, (hipStream_t)stream) == hipSuccess ? FA_OK : FA_ERR_DEVICE;
}

extern "C" int64_t fa_layer_norm_backward_workspace(const int64_t* sizes_host, int p, int features) {
  fa_row_blocks b;
  if (!row_blocks(sizes_host, p, &b) || features < 1 || features > FA_NORM_FEATURES_MAX) return -1;
  return (int64_t)fa_layer_norm_partials(b, b.row0[p], features);
}

extern "C" fa_status fa_layer_norm_backward(const void* dy, int64_t lddy, const int64_t* sizes_host, int p, int features,
                                            int dtype, const void* x, int64_t ldx, const float* mean, const float* rstd,
                                            const int8_t* codes, const uint8_t* exponents, const void* gamma, int param_dtype,
                                            const void* residual, int64_t ldr, void* dx, int64_t lddx, void* dgamma,
                                            int64_t lddgamma, void* dbeta, int64_t lddbeta, int grad_dtype, void* workspace,
                                            int64_t workspace_bytes, void* stream) {
  fa_norm_grad_args a;
  if (!known(dtype) || !known(param_dtype) || !known(grad_dtype) || !row_blocks(sizes_host, p, &a.blocks) ||
      !extent(0, features, FA_NORM_FEATURES_MAX))
    return FA_ERR_ARG;
  const int64_t rows = a.blocks.row0[p];
  if (!matrix(dy, lddy, rows, features, dtype) || !matrix(dx, lddx, rows, features, dtype) || !params(gamma, param_dtype) ||
      !floats(mean) || !floats(rstd) || (rows > 0 && !rstd))
    return FA_ERR_ARG;
  // xhat: from x with its statistics, or from the checkpoint, one of the two
  if (rows > 0 && ((x == nullptr) == (codes == nullptr) || (x && !mean))) return FA_ERR_ARG;
  if (x && !matrix(x, ldx, rows, features, dtype)) return FA_ERR_ARG;
  if (codes && !checkpoint(codes, exponents, rows)) return FA_ERR_ARG;
  if (residual && !matrix(residual, ldr, rows, features, dtype)) return FA_ERR_ARG;
  if (rows > 0 && (dx == dy || dx == x || dx == residual)) return FA_ERR_ARG;
  if (dgamma && !matrix(dgamma, lddgamma, p, features, grad_dtype)) return FA_ERR_ARG;
  if (dbeta && !matrix(dbeta, lddbeta, p, features, grad_dtype)) return FA_ERR_ARG;
  if (dgamma || dbeta) {
    const int64_t need = (int64_t)fa_layer_norm_partials(a.blocks, rows, features);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < need)) return FA_ERR_ARG;
  }
  a.dy = dy; a.x = x; a.gamma = gamma; a.residual = residual;
  a.mean = mean; a.rstd = rstd; a.codes = codes; a.exponents = exponents;
  a.dx = dx; a.dgamma = dgamma; a.dbeta = dbeta; a.partials = static_cast<float*>(workspace);
  a.lddy = lddy; a.ldx = ldx; a.ldr = ldr; a.lddx = lddx; a.lddgamma = lddgamma; a.lddbeta = lddbeta; a.rows = rows;
  a.features = features; a.param_bf16 = param_dtype == FA_BF16; a.grad_bf16 = grad_dtype == FA_BF16;
  return fa_launch_layer_norm_backward(a, dtype, (hipStream_t)stream) == hipSuccess ? FA_OK : FA_ERR_DEVICE;
}

extern "C" int64_t fa_linear_grad_workspace(const int64_t* sizes_host, int p, int features, int outputs, int dtype) {
  fa_row_blocks b;
  if (!known(dtype) || !row_blocks(sizes_host, p, &b) || !extent(0, features, FA_FEATURES_MAX) ||
      !extent(0, outputs, FA_FEATURES_MAX))
    return -1;
  return (int64_t)fa_linear_grad_partials(b, features, outputs, dtype);
}

extern "C" fa_status fa_linear_grad(const void* dy, int64_t lddy, const int64_t* sizes_host, int p, int features, int outputs,
                                    int dtype, const int8_t* codes, const uint8_t* exponents, const void* gamma,
                                    const void* beta, int param_dtype, void* dweight, int64_t lddweight, void* dbias,
                                    int64_t lddbias, int grad_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
  fa_linear_grad_args a;
  if (!known(dtype) || !known(param_dtype) || !known(grad_dtype) || !row_blocks(sizes_host, p, &a.blocks) ||
      !extent(0, features, FA_FEATURES_MAX) || !extent(0, outputs, FA_FEATURES_MAX))
    return FA_ERR_ARG;
  const int64_t rows = a.blocks.row0[p];
  if (!matrix(dy, lddy, rows, outputs, dtype) || !checkpoint(codes, exponents, rows) ||
      (gamma == nullptr) != (beta == nullptr) || !params(gamma, param_dtype) || !params(beta, param_dtype) ||
      !matrix(dweight, lddweight, p, (int64_t)outputs * features, grad_dtype) ||
      (dbias && !matrix(dbias, lddbias, p, outputs, grad_dtype)))
    return FA_ERR_ARG;
  const int64_t need = (int64_t)fa_linear_grad_partials(a.blocks, features, outputs, dtype);
  if (need > 0 && (!workspace || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < need)) return FA_ERR_ARG;
  a.dy = dy; a.gamma = gamma; a.beta = beta; a.codes = codes; a.exponents = exponents;
  a.dweight = dweight; a.dbias = dbias; a.partials = static_cast<float*>(workspace);
  // (rows that a step lacks are past the end of its buffer.  The pitch of a single row, or of none, has no meaning to the
  // caller and may be 0, which would put them inside that row)
  a.lddy = rows <= 1 ? outputs : lddy; a.lddweight = lddweight; a.lddbias = lddbias;
  a.features = features; a.outputs = outputs; a.splits = 1; a.param_bf16 = param_dtype == FA_BF16; a.grad_bf16 = grad_dtype == FA_BF16;
  return fa_launch_linear_grad(a, dtype, (hipStream_t)stream) == hipSuccess ? FA_OK : FA_ERR_DEVICE;
}
