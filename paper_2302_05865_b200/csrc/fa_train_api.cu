// C ABI of the training operators (declared in include/fa.h): argument checks, workspace carving, launches.
// Nothing here allocates, frees or synchronises.
#include <math.h>
#include <stdint.h>

#include "../../include/fa.h"
#include "fa_act8.cuh"
#include "fa_train.h"

namespace fa {
namespace {

constexpr size_t kWsAlign = 256;
inline size_t ws_round(size_t v) { return (v + kWsAlign - 1) / kWsAlign * kWsAlign; }

bool type_ok(int dtype) { return dtype == FA_F32 || dtype == FA_BF16; }
size_t size_of(int dtype) { return dtype == FA_F32 ? 4 : 2; }
bool at(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool size_ok(long long rows, long long cols) {
  return rows >= 0 && rows <= FA_MAX_ROWS && cols >= 1 && cols <= FA_MAX_COLS;
}
// A matrix that is read: any row stride that keeps addresses in range (0: one row for all).
bool in_ok(const void* p, long long ld, long long rows) {
  return rows == 0 || (p && ld >= 0 && ld <= (1LL << 40));
}
// A matrix that is written: rows must not overlap.
bool out_ok(const void* p, long long ld, long long rows, long long cols) {
  return rows == 0 || (p && (ld >= cols || rows == 1) && ld >= 0 && ld <= (1LL << 40));
}

int cuda_code(cudaError_t e) { return e == cudaSuccess ? FA_OK : FA_ERR_CUDA; }

// A product: tokens are counted in 32 bits on the device, and the result has to fit some memory.
bool product_ok(long long rows, long long outs, long long ins) {
  return size_ok(rows, outs) && size_ok(rows, ins) && rows <= FA_MAX_TOKENS && outs * ins <= (1LL << 40);
}
size_t layer_norm_ws(long long rows, long long cols, size_t* stats_at) {
  const size_t partials = ws_round(layer_norm_partials_bytes(rows, cols));
  if (stats_at) *stats_at = partials;
  return partials + (layer_norm_needs_row_stats(cols) ? ws_round((size_t)rows * 2 * sizeof(float)) : 0);
}
}  // namespace
}  // namespace fa

extern "C" {

int fa_checkpoint8_bytes(long long rows, long long cols, size_t* bytes) {
  if (!bytes || !fa::size_ok(rows, cols)) return FA_ERR_ARG;
  *bytes = fa::act8_scale_offset(rows, cols) + fa::ws_round((size_t)(rows * fa::act8_scale_pitch(cols)));
  return FA_OK;
}

int fa_checkpoint8_store(const void* x, long long ldx, int dtype, long long rows, long long cols, void* ck,
                         void* stream) {
  if (!fa::type_ok(dtype) || !fa::size_ok(rows, cols) || !fa::in_ok(x, ldx, rows)) return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  if (!ck) return FA_ERR_ARG;
  if (!fa::at(x, fa::size_of(dtype)) || !fa::at(ck, 16)) return FA_ERR_ALIGN;
  return fa::cuda_code(fa::launch_act8_store({x, ldx}, dtype, rows, cols, ck, static_cast<cudaStream_t>(stream)));
}

int fa_checkpoint8_load(const void* ck, int dtype, long long rows, long long cols, void* out, long long ldo,
                        void* stream) {
  if (!fa::type_ok(dtype) || !fa::size_ok(rows, cols) || !fa::out_ok(out, ldo, rows, cols)) return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  if (!ck) return FA_ERR_ARG;
  if (!fa::at(out, fa::size_of(dtype)) || !fa::at(ck, 16)) return FA_ERR_ALIGN;
  return fa::cuda_code(fa::launch_act8_load(ck, rows, cols, {out, ldo}, dtype, static_cast<cudaStream_t>(stream)));
}

int fa_gelu_forward(const void* x, long long ldx, int dtype, long long rows, long long cols, const void* bias,
                    int pdtype, int approximate, void* y, long long ldy, void* ck_x, void* ck_y, void* stream) {
  if (!fa::type_ok(dtype) || !fa::size_ok(rows, cols) || !fa::in_ok(x, ldx, rows) || !fa::out_ok(y, ldy, rows, cols) ||
      (bias && !fa::type_ok(pdtype)) || (approximate != FA_GELU_ERF && approximate != FA_GELU_TANH))
    return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  const size_t e = fa::size_of(dtype);
  if (!fa::at(x, e) || !fa::at(y, e) || (bias && !fa::at(bias, fa::size_of(pdtype))) || (ck_x && !fa::at(ck_x, 16)) ||
      (ck_y && !fa::at(ck_y, 16)))
    return FA_ERR_ALIGN;
  return fa::cuda_code(fa::launch_gelu_forward({x, ldx}, dtype, rows, cols, {bias, pdtype}, approximate, {y, ldy}, ck_x,
                                               ck_y, static_cast<cudaStream_t>(stream)));
}

int fa_gelu_backward_workspace_bytes(long long rows, long long cols, size_t* bytes) {
  if (!bytes || !fa::size_ok(rows, cols)) return FA_ERR_ARG;
  *bytes = fa::ws_round(fa::column_partials_bytes(rows, cols));
  return FA_OK;
}

int fa_gelu_backward(const void* dy, long long lddy, const void* x, long long ldx, const void* bias, int pdtype,
                     const void* ck, int dtype, long long rows, long long cols, int approximate, void* dx,
                     long long lddx, void* dbias, int gdtype, void* ws, size_t ws_bytes, void* stream) {
  if (!fa::type_ok(dtype) || !fa::size_ok(rows, cols) || !fa::in_ok(dy, lddy, rows) ||
      !fa::out_ok(dx, lddx, rows, cols) || (approximate != FA_GELU_ERF && approximate != FA_GELU_TANH) ||
      (bias && !fa::type_ok(pdtype)) || (dbias && (!fa::type_ok(gdtype) || !ws)))
    return FA_ERR_ARG;
  // the input comes from exactly one place; a checkpoint holds it with the bias in it
  if (rows > 0 && ((ck != nullptr) == (x != nullptr) || (ck && bias) || (x && !fa::in_ok(x, ldx, rows)))) return FA_ERR_ARG;
  const size_t e = fa::size_of(dtype);
  if (!fa::at(dy, e) || !fa::at(x, e) || !fa::at(dx, e) || (bias && !fa::at(bias, fa::size_of(pdtype))) ||
      !fa::at(ck, 16) || (dbias && (!fa::at(dbias, fa::size_of(gdtype)) || !fa::at(ws, 16))))
    return FA_ERR_ALIGN;
  if (dbias && ws_bytes < fa::ws_round(fa::column_partials_bytes(rows, cols))) return FA_ERR_WORKSPACE;
  return fa::cuda_code(fa::launch_gelu_backward({dy, lddy}, {x, ldx}, {bias, pdtype}, ck, dtype, rows, cols, approximate,
                                                {dx, lddx}, dbias, gdtype, static_cast<float*>(ws),
                                                static_cast<cudaStream_t>(stream)));
}

int fa_layer_norm_forward(const void* x, long long ldx, const void* residual, long long ldr, int dtype, long long rows,
                          long long cols, const void* weight, const void* bias, int pdtype, float eps, void* y,
                          long long ldy, void* sum_out, long long lds, float* mean, float* rstd, void* ck_sum,
                          void* ck_y, void* stream) {
  if (!fa::type_ok(dtype) || !fa::size_ok(rows, cols) || !fa::in_ok(x, ldx, rows) || !fa::out_ok(y, ldy, rows, cols) ||
      ((weight || bias) && !fa::type_ok(pdtype)) || !(eps >= 0.f) || isinf(eps) ||
      (residual && !fa::in_ok(residual, ldr, rows)) || (sum_out && !fa::out_ok(sum_out, lds, rows, cols)))
    return FA_ERR_ARG;
  if (rows == 0) return FA_OK;
  const size_t e = fa::size_of(dtype);
  if (!fa::at(x, e) || !fa::at(residual, e) || !fa::at(y, e) || !fa::at(sum_out, e) ||
      ((weight || bias) && (!fa::at(weight, fa::size_of(pdtype)) || !fa::at(bias, fa::size_of(pdtype)))) ||
      !fa::at(mean, 4) || !fa::at(rstd, 4) || !fa::at(ck_sum, 16) || !fa::at(ck_y, 16))
    return FA_ERR_ALIGN;
  return fa::cuda_code(fa::launch_layer_norm_forward({x, ldx}, {residual, ldr}, dtype, rows, cols, {weight, pdtype},
                                                     {bias, pdtype}, eps, {y, ldy}, {sum_out, lds}, mean, rstd, ck_sum,
                                                     ck_y, static_cast<cudaStream_t>(stream)));
}

int fa_layer_norm_backward_workspace_bytes(long long rows, long long cols, size_t* bytes) {
  if (!bytes || !fa::size_ok(rows, cols)) return FA_ERR_ARG;
  *bytes = fa::layer_norm_ws(rows, cols, nullptr);
  return FA_OK;
}

int fa_layer_norm_backward(const void* dy, long long lddy, const void* x, long long ldx, const void* ck, int dtype,
                           long long rows, long long cols, const void* weight, int pdtype, const float* mean,
                           const float* rstd, const void* residual_grad, long long ldr, void* dx, long long lddx,
                           void* dweight, void* dbias, int gdtype, void* ws, size_t ws_bytes, void* stream) {
  if (!fa::type_ok(dtype) || !fa::size_ok(rows, cols) || !fa::in_ok(dy, lddy, rows) ||
      !fa::out_ok(dx, lddx, rows, cols) || (weight && !fa::type_ok(pdtype)) ||
      ((dweight || dbias) && !fa::type_ok(gdtype)) || (residual_grad && !fa::in_ok(residual_grad, ldr, rows)) || !ws)
    return FA_ERR_ARG;
  if (rows > 0 && ((ck != nullptr) == (x != nullptr) || !mean || !rstd || (x && !fa::in_ok(x, ldx, rows))))
    return FA_ERR_ARG;
  const size_t e = fa::size_of(dtype);
  if (!fa::at(dy, e) || !fa::at(x, e) || !fa::at(residual_grad, e) || !fa::at(dx, e) ||
      (weight && !fa::at(weight, fa::size_of(pdtype))) || !fa::at(mean, 4) || !fa::at(rstd, 4) || !fa::at(ck, 16) ||
      ((dweight || dbias) && (!fa::at(dweight, fa::size_of(gdtype)) || !fa::at(dbias, fa::size_of(gdtype)))) ||
      !fa::at(ws, 16))
    return FA_ERR_ALIGN;
  size_t stats_at = 0;
  if (ws_bytes < fa::layer_norm_ws(rows, cols, &stats_at)) return FA_ERR_WORKSPACE;
  return fa::cuda_code(fa::launch_layer_norm_backward(
      {dy, lddy}, {x, ldx}, ck, dtype, rows, cols, {weight, pdtype}, mean, rstd, {residual_grad, ldr}, {dx, lddx},
      dweight, dbias, gdtype, static_cast<float*>(ws), reinterpret_cast<float*>(static_cast<char*>(ws) + stats_at),
      static_cast<cudaStream_t>(stream)));
}

int fa_linear_weight_grad_workspace_bytes(long long rows, long long outs, long long ins, int dtype, int aligned,
                                          size_t* bytes) {
  if (!bytes || !fa::type_ok(dtype) || !fa::product_ok(rows, outs, ins)) return FA_ERR_ARG;
  *bytes = fa::ws_round(fa::linear_weight_grad_scratch_bytes(rows, outs, ins, dtype, aligned && dtype == FA_BF16));
  return FA_OK;
}

int fa_linear_weight_grad(const void* dy, long long lddy, int dtype, long long rows, long long outs, const void* ck,
                          long long ins, void* dweight, void* dbias, int gdtype, void* ws, size_t ws_bytes,
                          void* stream) {
  if (!fa::type_ok(dtype) || !fa::type_ok(gdtype) || !fa::product_ok(rows, outs, ins) ||
      !fa::in_ok(dy, lddy, rows) || !dweight || !ws || (rows > 0 && !ck))
    return FA_ERR_ARG;
  if (!fa::at(dy, fa::size_of(dtype)) || !fa::at(ck, 16) || !fa::at(dweight, fa::size_of(gdtype)) ||
      !fa::at(dbias, fa::size_of(gdtype)) || !fa::at(ws, 16))
    return FA_ERR_ALIGN;
  const bool direct = fa::linear_weight_grad_direct({dy, lddy}, dtype, outs);
  if (ws_bytes < fa::linear_weight_grad_scratch_bytes(rows, outs, ins, dtype, direct)) return FA_ERR_WORKSPACE;
  return fa::cuda_code(fa::launch_linear_weight_grad({dy, lddy}, dtype, rows, outs, ins, ck, dweight, dbias, gdtype, ws,
                                                     static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
