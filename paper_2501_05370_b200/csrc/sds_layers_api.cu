// C entry points of the layer operators (see include/sds.h): argument checks and workspace carving.
#include "../../include/sds.h"

#include <cmath>

#include "sds_layers.h"

using namespace sds;

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxSize = (int64_t)1 << 30;   // of rows, d and f each: the kernels count them in 32 bits
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool is_type(int32_t t) { return t == SDS_F32 || t == SDS_BF16 || t == SDS_F16; }
inline size_t type_bytes(int32_t t) { return t == SDS_F32 ? 4 : 2; }

int result(cudaError_t e) {
  if (e == cudaSuccess) return SDS_OK;
  cudaGetLastError();
  return SDS_ECUDA;
}

int check_norm(int64_t rows, int32_t d, int32_t x_dtype, int32_t y_dtype, int32_t w_dtype) {
  if (rows < 0 || rows > kMaxSize || d <= 0 || d > kMaxSize) return SDS_EINVAL;
  if (!is_type(x_dtype) || !is_type(y_dtype) || !is_type(w_dtype)) return SDS_EUNSUPPORTED;
  if (y_dtype != x_dtype && x_dtype != SDS_F32) return SDS_EUNSUPPORTED;
  return SDS_OK;
}

// an array of rows: present and element-aligned unless there is nothing in it
int check_rows(const void* p, int64_t ld, int32_t dtype, int64_t rows, int32_t d) {
  if (rows == 0) return SDS_OK;
  if (!p || ld < d) return SDS_EINVAL;
  return aligned(p, type_bytes(dtype)) ? SDS_OK : SDS_EINVAL;
}

int check_workspace(const void* p, size_t have, size_t need) {
  return !p || have < need || !aligned(p, kAlign) ? SDS_ENOMEM : SDS_OK;
}

size_t norm_bytes(int64_t rows, int32_t d) {
  return align_up((size_t)norm_parts((int)rows, d) * 2 * (size_t)d * 4) +
         (norm_is_long(d) ? align_up((size_t)rows * 4) : 0) + kAlign;
}

int check_ffn(int64_t rows, int32_t d, int32_t f) {
  if (rows < 0 || rows > kMaxSize || d <= 0 || d > kMaxSize || f <= 0 || f > kMaxSize) return SDS_EINVAL;
  return d % 8 || f % 8 ? SDS_EUNSUPPORTED : SDS_OK;
}

// rows the tensor maps read or the 16-byte stores write
int check_ffn_rows(const void* p, int64_t ld, int64_t rows, int32_t d) {
  if (rows == 0) return SDS_OK;
  if (!p || ld < d) return SDS_EINVAL;
  return aligned(p, 16) && ld % 8 == 0 && ld < ((int64_t)1 << 38) ? SDS_OK : SDS_EUNSUPPORTED;
}

size_t hidden_bytes(int64_t rows, int32_t f) { return align_up((size_t)rows * f * 2); }
size_t factor_bytes(int64_t rows, int32_t f) { return align_up(ffn_keep_floats(rows, f) * 4); }

sds_gated_ffn_sizes ffn_sizes(int64_t rows, int32_t d, int32_t f) {
  sds_gated_ffn_sizes s;
  s.keep_bytes = factor_bytes(rows, f) + hidden_bytes(rows, f) + kAlign;
  s.forward_keep_bytes = kAlign;                       // the status word
  s.forward_bytes = kAlign + hidden_bytes(rows, f);
  s.backward_bytes = kAlign + 2 * hidden_bytes(rows, f) + align_up(ffn_part_floats(rows, d, f) * 4);
  return s;
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

int sds_layer_norm(const void* x_dev, int64_t ldx, int32_t x_dtype, const void* w_dev, const void* b_dev,
                   int32_t w_dtype, int64_t rows, int32_t d, float eps, void* y_dev, int64_t ldy, int32_t y_dtype,
                   float* mean_dev, float* rstd_dev, void* cuda_stream) {
  int rc = check_norm(rows, d, x_dtype, y_dtype, w_dtype);
  if (rc != SDS_OK) return rc;
  if (!std::isfinite(eps) || eps < 0.f) return SDS_EINVAL;
  if ((rc = check_rows(x_dev, ldx, x_dtype, rows, d)) != SDS_OK) return rc;
  if ((rc = check_rows(y_dev, ldy, y_dtype, rows, d)) != SDS_OK) return rc;
  if (!aligned(w_dev, type_bytes(w_dtype)) || !aligned(b_dev, type_bytes(w_dtype)) || !aligned(mean_dev, 4) ||
      !aligned(rstd_dev, 4))
    return SDS_EINVAL;
  NormArgs a{};
  a.x = x_dev; a.ldx = ldx; a.tx = x_dtype;
  a.w = w_dev; a.b = b_dev; a.tw = w_dtype;
  a.y = y_dev; a.ldy = ldy; a.ty = y_dtype;
  a.mean = mean_dev; a.rstd = rstd_dev;
  a.rows = (int)rows; a.d = d; a.eps = eps;
  return result(launch_norm(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_layer_norm_workspace_bytes(int64_t rows, int32_t d, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxSize || d <= 0 || d > kMaxSize) return SDS_EINVAL;
  *bytes = norm_bytes(rows, d);
  return SDS_OK;
}

int sds_layer_norm_backward(const void* dy_dev, int64_t lddy, int32_t y_dtype, const void* x_dev, int64_t ldx,
                            int32_t x_dtype, const void* w_dev, int32_t w_dtype, const float* mean_dev,
                            const float* rstd_dev, int64_t rows, int32_t d, void* dx_dev, int64_t lddx, void* dw_dev,
                            void* db_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_norm(rows, d, x_dtype, y_dtype, w_dtype);
  if (rc != SDS_OK) return rc;
  if ((rc = check_rows(dy_dev, lddy, y_dtype, rows, d)) != SDS_OK) return rc;
  if ((rc = check_rows(x_dev, ldx, x_dtype, rows, d)) != SDS_OK) return rc;
  if (dx_dev && (rc = check_rows(dx_dev, lddx, x_dtype, rows, d)) != SDS_OK) return rc;
  if (rows > 0 && (!mean_dev || !rstd_dev)) return SDS_EINVAL;
  if (!aligned(w_dev, type_bytes(w_dtype)) || !aligned(dw_dev, type_bytes(w_dtype)) ||
      !aligned(db_dev, type_bytes(w_dtype)) || !aligned(mean_dev, 4) || !aligned(rstd_dev, 4))
    return SDS_EINVAL;
  if ((rc = check_workspace(workspace_dev, workspace_bytes, norm_bytes(rows, d))) != SDS_OK) return rc;
  if (!dx_dev && !dw_dev && !db_dev) return SDS_OK;
  NormArgs a{};
  a.dy = dy_dev; a.lddy = lddy; a.ty = y_dtype;
  a.x = x_dev; a.ldx = ldx; a.tx = x_dtype;
  a.w = w_dev; a.tw = w_dtype;
  a.mean = const_cast<float*>(mean_dev); a.rstd = const_cast<float*>(rstd_dev);
  a.rows = (int)rows; a.d = d;
  a.dx = dx_dev; a.lddx = lddx; a.dw = dw_dev; a.db = db_dev;
  a.part = static_cast<float*>(workspace_dev);
  a.shift = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) +
                                     align_up((size_t)norm_parts((int)rows, d) * 2 * (size_t)d * 4));
  return result(launch_norm_backward(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_gated_ffn_bytes(int64_t rows, int32_t d, int32_t f, sds_gated_ffn_sizes* sizes) {
  if (!sizes) return SDS_EINVAL;
  const int rc = check_ffn(rows, d, f);
  if (rc != SDS_OK) return rc;
  *sizes = ffn_sizes(rows, d, f);
  return SDS_OK;
}

int sds_gated_ffn(const void* x_dev, int64_t ldx, int32_t dtype, int64_t rows, int32_t d, int32_t f,
                  const void* wg_dev, const void* wu_dev, const void* wd_dev, int32_t act, void* y_dev, int64_t ldy,
                  void* keep_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_ffn(rows, d, f);
  if (rc != SDS_OK) return rc;
  if (dtype != SDS_BF16 && dtype != SDS_F16) return SDS_EUNSUPPORTED;
  if (act != SDS_ACT_SILU && act != SDS_ACT_GELU && act != SDS_ACT_GELU_TANH) return SDS_EUNSUPPORTED;
  if (!wg_dev || !wu_dev || !wd_dev) return SDS_EINVAL;
  if (!aligned(wg_dev, 16) || !aligned(wu_dev, 16) || !aligned(wd_dev, 16)) return SDS_EUNSUPPORTED;
  if ((rc = check_ffn_rows(x_dev, ldx, rows, d)) != SDS_OK) return rc;
  if ((rc = check_ffn_rows(y_dev, ldy, rows, d)) != SDS_OK) return rc;
  const sds_gated_ffn_sizes s = ffn_sizes(rows, d, f);
  if ((rc = check_workspace(workspace_dev, workspace_bytes, keep_dev ? s.forward_keep_bytes : s.forward_bytes)) != SDS_OK)
    return rc;
  if (!aligned(keep_dev, kAlign)) return SDS_ENOMEM;
  FfnArgs a{};
  a.rows = (int)rows; a.d = d; a.f = f;
  a.f16 = dtype == SDS_F16; a.act = act;
  a.x = x_dev; a.ldx = ldx; a.y = y_dev; a.ldy = ldy;
  a.wg = wg_dev; a.wu = wu_dev; a.wd = wd_dev;
  a.err = static_cast<int*>(workspace_dev);
  a.keep = static_cast<float*>(keep_dev);
  a.h = keep_dev ? static_cast<char*>(keep_dev) + factor_bytes(rows, f) : static_cast<char*>(workspace_dev) + kAlign;
  return result(launch_ffn(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_gated_ffn_backward(const void* dy_dev, int64_t lddy, const void* x_dev, int64_t ldx, int32_t dtype,
                           int64_t rows, int32_t d, int32_t f, const void* wg_dev, const void* wu_dev,
                           const void* wd_dev, const void* keep_dev, void* dx_dev, int64_t lddx, void* dwg_dev,
                           void* dwu_dev, void* dwd_dev, void* workspace_dev, size_t workspace_bytes,
                           void* cuda_stream) {
  int rc = check_ffn(rows, d, f);
  if (rc != SDS_OK) return rc;
  if (dtype != SDS_BF16 && dtype != SDS_F16) return SDS_EUNSUPPORTED;
  if (!wg_dev || !wu_dev || !wd_dev) return SDS_EINVAL;
  for (const void* p : {wg_dev, wu_dev, wd_dev, (const void*)dwg_dev, (const void*)dwu_dev, (const void*)dwd_dev})
    if (!aligned(p, 16)) return SDS_EUNSUPPORTED;
  if ((rc = check_ffn_rows(dy_dev, lddy, rows, d)) != SDS_OK) return rc;
  if ((rc = check_ffn_rows(x_dev, ldx, rows, d)) != SDS_OK) return rc;
  if (dx_dev && (rc = check_ffn_rows(dx_dev, lddx, rows, d)) != SDS_OK) return rc;
  if (rows > 0 && !keep_dev) return SDS_EINVAL;
  if (!aligned(keep_dev, kAlign)) return SDS_ENOMEM;
  if ((rc = check_workspace(workspace_dev, workspace_bytes, ffn_sizes(rows, d, f).backward_bytes)) != SDS_OK) return rc;
  FfnArgs a{};
  a.rows = (int)rows; a.d = d; a.f = f;
  a.f16 = dtype == SDS_F16;
  a.x = x_dev; a.ldx = ldx; a.dy = dy_dev; a.lddy = lddy;
  a.wg = wg_dev; a.wu = wu_dev; a.wd = wd_dev;
  a.dx = dx_dev; a.lddx = lddx; a.dwg = dwg_dev; a.dwu = dwu_dev; a.dwd = dwd_dev;
  char* ws = static_cast<char*>(workspace_dev);
  a.err = reinterpret_cast<int*>(ws);
  a.dg = ws + kAlign;
  a.du = ws + kAlign + hidden_bytes(rows, f);
  a.part = reinterpret_cast<float*>(ws + kAlign + 2 * hidden_bytes(rows, f));
  a.keep = static_cast<float*>(const_cast<void*>(keep_dev));
  a.h = static_cast<char*>(const_cast<void*>(keep_dev)) + factor_bytes(rows, f);
  return result(launch_ffn_backward(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_gated_ffn_status(const void* workspace_dev, void* cuda_stream) {
  if (!workspace_dev) return SDS_EINVAL;
  int word = 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaMemcpyAsync(&word, workspace_dev, sizeof(word), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return result(e);
  return word != 0 ? SDS_ETIMEOUT : SDS_OK;
}

int sds_gated_ffn_gave_up(void* cuda_stream) {
  int role = 0;
  const cudaError_t e = ffn_gave_up(&role, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return result(e);
  return role != 0 ? SDS_ETIMEOUT : SDS_OK;
}

int sds_selftest_gated_ffn_wait(int32_t polls, void* workspace_dev, void* cuda_stream) {
  if (!workspace_dev || !aligned(workspace_dev, kAlign) || polls <= 0 || polls > (1 << 16)) return SDS_EINVAL;
  return result(launch_ffn_wait_selftest((uint32_t)polls, static_cast<int*>(workspace_dev), static_cast<cudaStream_t>(cuda_stream)));
}

#pragma GCC visibility pop
}  // extern "C"
