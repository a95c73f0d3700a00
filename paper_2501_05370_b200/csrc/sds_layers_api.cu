// C entry points of the layer operators (see include/sds.h): argument checks and workspace carving.
#include "../../include/sds.h"

#include <algorithm>
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

int check_linear(const sds_linear_layer* l, int64_t rows) {
  if (!l || rows < 0 || rows > kMaxSize || l->k <= 0 || l->k > kMaxSize || l->n <= 0 || l->n > kMaxSize) return SDS_EINVAL;
  if (l->table_dev ? l->steps <= 0 : l->steps < 0) return SDS_EINVAL;
  if (l->dtype != SDS_BF16 && l->dtype != SDS_F16) return SDS_EUNSUPPORTED;
  if (l->act != SDS_ACT_NONE && l->act != SDS_ACT_SILU && l->act != SDS_ACT_GELU && l->act != SDS_ACT_GELU_TANH)
    return SDS_EUNSUPPORTED;
  return l->k % 8 || (l->table_dev && l->steps > 65535) ? SDS_EUNSUPPORTED : SDS_OK;
}

// the layer's arrays, and what both directions read
int check_linear_call(const sds_linear_layer* l, const void* x, int64_t ldx, const int32_t* step, int64_t rows, int32_t y_dtype) {
  int rc = check_linear(l, rows);
  if (rc != SDS_OK) return rc;
  if (y_dtype != SDS_F32 && y_dtype != l->dtype) return SDS_EUNSUPPORTED;
  if (!l->w_dev) return SDS_EINVAL;
  if (!aligned(l->w_dev, 16)) return SDS_EUNSUPPORTED;
  if (l->bias_dev && (!is_type(l->bias_dtype) || !aligned(l->bias_dev, type_bytes(l->bias_dtype))))
    return is_type(l->bias_dtype) ? SDS_EINVAL : SDS_EUNSUPPORTED;
  if (!aligned(l->table_dev, 2)) return SDS_EINVAL;
  if (l->table_dev && rows > 0 && (!step || !aligned(step, 4))) return SDS_EINVAL;
  return check_ffn_rows(x, ldx, rows, l->k);
}

sds_linear_sizes linear_sizes(const sds_linear_layer* l, int64_t rows) {
  sds_linear_sizes s;
  s.keep_bytes = l->act == SDS_ACT_NONE ? 0 : align_up(linear_factor_bytes(rows, l->n));
  s.forward_bytes = kAlign;                            // the status word
  s.backward_bytes = linear_workspace(rows, l->k, l->n, l->steps, l->table_dev != nullptr).bytes;
  return s;
}

LinearArgs linear_args(const sds_linear_layer* l, const void* x, int64_t ldx, const int32_t* step, int64_t rows, int32_t y_dtype,
                       const void* keep, void* workspace) {
  LinearArgs a{};
  a.rows = (int)rows; a.k = l->k; a.n = l->n;
  a.f16 = l->dtype == SDS_F16; a.act = l->act;
  a.x = x; a.ldx = ldx; a.w = l->w_dev;
  a.bias = l->bias_dev; a.tbias = l->bias_dtype;
  a.table = l->table_dev; a.step = step; a.steps = l->steps;
  a.ty = y_dtype;
  a.factor = static_cast<float*>(const_cast<void*>(keep));
  a.err = static_cast<int*>(workspace);
  return a;
}

int check_dropout(const sds_dropout_spec& s, int64_t rows) {
  constexpr int64_t kMostRows = (int64_t)1 << 56;
  if (!(s.p >= 0.0 && s.p <= 1.0) || s.step < 0 || s.row0 < 0 || s.row0 > kMostRows - rows || !aligned(s.step_dev, 4)) return SDS_EINVAL;
  return SDS_OK;
}

DropoutArgs dropout_args(const sds_dropout_spec& s) {
  DropoutArgs a{};
  a.threshold = (uint32_t)std::nearbyint(s.p * 65536.0);
  a.scale = a.threshold < 65536u ? (float)(65536.0 / (65536.0 - a.threshold)) : 0.f;
  a.seed = s.seed; a.step = (uint32_t)s.step; a.step_dev = s.step_dev; a.row0 = (uint64_t)s.row0;
  return a;
}

// rows that the residual norm's kernels reach by one 32-bit multiplication
int check_near_rows(const void* p, int64_t ld, int32_t dtype, int64_t rows, int32_t d) {
  const int rc = check_rows(p, ld, dtype, rows, d);
  return rc != SDS_OK || rows == 0 ? rc : ld < ((int64_t)1 << 31) ? SDS_OK : SDS_EUNSUPPORTED;
}
// a vector per group
int check_cond(const void* p, int64_t ld, int32_t type, int64_t groups, int32_t d) { return p ? check_near_rows(p, ld, type, groups, d) : SDS_OK; }

int check_residual_norm(const sds_residual_norm_op* op) {
  if (!op || op->rows < 0 || op->rows > kMaxSize || op->d <= 0 || op->groups < 1 || (op->rows > 0 && op->rows % op->groups) ||
      (op->rows == 0 && op->groups > kMaxSize))
    return SDS_EINVAL;
  if (op->kind != SDS_NORM_LAYER && op->kind != SDS_NORM_RMS) return SDS_EINVAL;
  if (!std::isfinite(op->eps) || op->eps < 0.f || !std::isfinite(op->alpha)) return SDS_EINVAL;
  if (op->d > kResidualMaxD) return SDS_EUNSUPPORTED;
  if (!is_type(op->r_dtype) || !is_type(op->h_dtype) || !is_type(op->w_dtype) || !is_type(op->cond_dtype)) return SDS_EUNSUPPORTED;
  if (op->h_dtype != op->r_dtype && op->r_dtype != SDS_F32) return SDS_EUNSUPPORTED;
  for (const void* p : {op->w_dev, op->b_dev, op->post_w_dev})
    if (!aligned(p, type_bytes(op->w_dtype))) return SDS_EINVAL;
  int rc;
  if ((rc = check_cond(op->gate_dev, op->ld_gate, op->cond_dtype, op->groups, op->d)) != SDS_OK) return rc;
  if ((rc = check_cond(op->scale_dev, op->ld_scale, op->cond_dtype, op->groups, op->d)) != SDS_OK) return rc;
  if ((rc = check_cond(op->shift_dev, op->ld_shift, op->cond_dtype, op->groups, op->d)) != SDS_OK) return rc;
  return check_dropout(op->drop, op->rows);
}

ResidualNormArgs residual_norm_args(const sds_residual_norm_op* op, const void* r, int64_t ldr, const void* h, int64_t ldh, const float* keep) {
  ResidualNormArgs a{};
  a.rows = (int)op->rows; a.d = op->d; a.groups = (int)op->groups; a.per = op->rows > 0 ? (int)(op->rows / op->groups) : 1;
  a.tr = op->r_dtype; a.th = op->h_dtype;
  a.rms = op->kind == SDS_NORM_RMS; a.post = h && op->post != 0;
  a.alpha = op->alpha; a.eps = op->eps;
  a.drop = dropout_args(op->drop);
  a.r = r; a.ldr = ldr; a.h = h; a.ldh = ldh;
  a.w = op->w_dev; a.b = op->b_dev; a.wp = a.post ? op->post_w_dev : nullptr; a.tw = op->w_dtype;
  a.gate = h ? op->gate_dev : nullptr; a.scale = op->scale_dev; a.shift = op->shift_dev; a.tc = op->cond_dtype;
  a.ldgate = op->ld_gate; a.ldscale = op->ld_scale; a.ldshift = op->ld_shift;
  a.stats = reinterpret_cast<float4*>(const_cast<float*>(keep));
  return a;
}

// the workspace of a backward call that wants the gradients of all that op has
size_t residual_norm_bytes(const sds_residual_norm_op* op) {
  if (op->rows == 0) return kAlign;
  size_t most = 0;
  for (const bool cond : {false, true}) {
    ResidualNormArgs a = residual_norm_args(op, nullptr, 0, op, 0, nullptr);    // (as if there were an h)
    a.dgate = cond ? &most : nullptr;
    size_t part = 0, groups = 0;
    residual_norm_plan(&a, &part, &groups);
    most = std::max(most, align_up(part * 4) + align_up(groups * 4));
  }
  return most;
}

int status_word(const void* workspace, void* cuda_stream) {
  if (!workspace) return SDS_EINVAL;
  int word = 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return result(e);
  return word != 0 ? SDS_ETIMEOUT : SDS_OK;
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

int sds_gated_ffn_status(const void* workspace_dev, void* cuda_stream) { return status_word(workspace_dev, cuda_stream); }

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

int sds_linear_bytes(const sds_linear_layer* layer, int64_t rows, sds_linear_sizes* sizes) {
  if (!sizes) return SDS_EINVAL;
  const int rc = check_linear(layer, rows);
  if (rc != SDS_OK) return rc;
  *sizes = linear_sizes(layer, rows);
  return SDS_OK;
}

int sds_linear(const sds_linear_layer* layer, const void* x_dev, int64_t ldx, const int32_t* step_dev, int64_t rows,
               const void* residual_dev, int64_t ldr, void* y_dev, int64_t ldy, int32_t y_dtype, void* keep_dev,
               void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_linear_call(layer, x_dev, ldx, step_dev, rows, y_dtype);
  if (rc != SDS_OK) return rc;
  if ((rc = check_rows(y_dev, ldy, y_dtype, rows, layer->n)) != SDS_OK) return rc;
  if (residual_dev && (rc = check_rows(residual_dev, ldr, y_dtype, rows, layer->n)) != SDS_OK) return rc;
  if ((rc = check_workspace(workspace_dev, workspace_bytes, kAlign)) != SDS_OK) return rc;
  if (!aligned(keep_dev, kAlign)) return SDS_ENOMEM;
  LinearArgs a = linear_args(layer, x_dev, ldx, step_dev, rows, y_dtype, keep_dev, workspace_dev);
  a.residual = residual_dev; a.ldr = ldr;
  a.y = y_dev; a.ldy = ldy;
  return result(launch_linear(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_linear_backward(const sds_linear_layer* layer, const void* dy_dev, int64_t lddy, int32_t y_dtype,
                        const void* x_dev, int64_t ldx, const int32_t* step_dev, int64_t rows, const void* keep_dev,
                        void* dx_dev, int64_t lddx, void* dw_dev, void* dbias_dev, void* dtable_dev,
                        void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_linear_call(layer, x_dev, ldx, step_dev, rows, y_dtype);
  if (rc != SDS_OK) return rc;
  if ((rc = check_rows(dy_dev, lddy, y_dtype, rows, layer->n)) != SDS_OK) return rc;
  if (dx_dev && (rc = check_ffn_rows(dx_dev, lddx, rows, layer->k)) != SDS_OK) return rc;
  if ((dbias_dev && !layer->bias_dev) || (dtable_dev && !layer->table_dev)) return SDS_EINVAL;
  if (dtable_dev && rows * layer->steps > ((int64_t)1 << 36)) return SDS_EUNSUPPORTED;     // (every step looks at every row's)
  if (!aligned(dw_dev, 16)) return SDS_EUNSUPPORTED;
  if ((dbias_dev && !aligned(dbias_dev, type_bytes(layer->bias_dtype))) || !aligned(dtable_dev, 2)) return SDS_EINVAL;
  const sds_linear_sizes s = linear_sizes(layer, rows);
  if (s.keep_bytes > 0 && !keep_dev) return SDS_EINVAL;
  if (!aligned(keep_dev, kAlign)) return SDS_ENOMEM;
  if ((rc = check_workspace(workspace_dev, workspace_bytes, s.backward_bytes)) != SDS_OK) return rc;
  LinearArgs a = linear_args(layer, x_dev, ldx, step_dev, rows, y_dtype, keep_dev, workspace_dev);
  a.dy = dy_dev; a.lddy = lddy;
  a.dx = dx_dev; a.lddx = lddx;
  a.dw = dw_dev; a.db = dbias_dev; a.dtable = dtable_dev;
  return result(launch_linear_backward(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_linear_status(const void* workspace_dev, void* cuda_stream) { return status_word(workspace_dev, cuda_stream); }

int sds_linear_gave_up(void* cuda_stream) {
  int role = 0;
  const cudaError_t e = linear_gave_up(&role, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return result(e);
  return role != 0 ? SDS_ETIMEOUT : SDS_OK;
}

int sds_dropout(const sds_dropout_spec* spec, const void* x_dev, int64_t ldx, int32_t x_dtype, int64_t rows, int32_t d,
                const void* residual_dev, int64_t ldr, void* y_dev, int64_t ldy, int32_t y_dtype, void* cuda_stream) {
  if (!spec || rows < 0 || rows > kMaxSize || d <= 0 || d > kMaxSize) return SDS_EINVAL;
  int rc = check_dropout(*spec, rows);
  if (rc != SDS_OK) return rc;
  if (!is_type(x_dtype) || !is_type(y_dtype) || (x_dtype != y_dtype && x_dtype != SDS_F32 && y_dtype != SDS_F32)) return SDS_EUNSUPPORTED;
  if ((rc = check_rows(x_dev, ldx, x_dtype, rows, d)) != SDS_OK) return rc;
  if ((rc = check_rows(y_dev, ldy, y_dtype, rows, d)) != SDS_OK) return rc;
  if (residual_dev && (rc = check_rows(residual_dev, ldr, y_dtype, rows, d)) != SDS_OK) return rc;
  DropoutCall a{};
  a.drop = dropout_args(*spec);
  a.x = x_dev; a.ldx = ldx; a.tx = x_dtype;
  a.residual = residual_dev; a.ldr = ldr;
  a.y = y_dev; a.ldy = ldy; a.ty = y_dtype;
  a.rows = rows; a.d = d;
  return result(launch_dropout(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_residual_norm(const sds_residual_norm_op* op, const void* r_dev, int64_t ldr, const void* h_dev, int64_t ldh,
                      void* out_dev, int64_t ldo, void* n_dev, int64_t ldn, float* keep_dev, void* cuda_stream) {
  int rc = check_residual_norm(op);
  if (rc != SDS_OK) return rc;
  if ((rc = check_near_rows(r_dev, ldr, op->r_dtype, op->rows, op->d)) != SDS_OK) return rc;
  if (h_dev && (rc = check_near_rows(h_dev, ldh, op->h_dtype, op->rows, op->d)) != SDS_OK) return rc;
  if (h_dev && (rc = check_near_rows(out_dev, ldo, op->r_dtype, op->rows, op->d)) != SDS_OK) return rc;
  if ((rc = check_near_rows(n_dev, ldn, op->h_dtype, op->rows, op->d)) != SDS_OK) return rc;
  if (!aligned(keep_dev, kAlign)) return SDS_ENOMEM;
  ResidualNormArgs a = residual_norm_args(op, r_dev, ldr, h_dev, ldh, keep_dev);
  a.out = out_dev; a.ldo = ldo;
  a.n = n_dev; a.ldn = ldn;
  return result(launch_residual_norm(a, static_cast<cudaStream_t>(cuda_stream)));
}

int sds_residual_norm_bytes(const sds_residual_norm_op* op, sds_residual_norm_sizes* sizes) {
  if (!sizes) return SDS_EINVAL;
  const int rc = check_residual_norm(op);
  if (rc != SDS_OK) return rc;
  sizes->keep_bytes = (size_t)op->rows * 8 * 4;
  sizes->backward_bytes = residual_norm_bytes(op);
  return SDS_OK;
}

int sds_residual_norm_backward(const sds_residual_norm_op* op, const void* dn_dev, int64_t lddn, const void* dout_dev,
                               int64_t lddout, const void* r_dev, int64_t ldr, const void* h_dev, int64_t ldh,
                               const float* keep_dev, const sds_residual_norm_grads* grads, void* workspace_dev,
                               size_t workspace_bytes, void* cuda_stream) {
  int rc = check_residual_norm(op);
  if (rc != SDS_OK) return rc;
  if (!grads) return SDS_EINVAL;
  const sds_residual_norm_grads& g = *grads;
  const struct { const void* p; int64_t ld; int32_t type; bool needed; } arrays[6] = {
      {dn_dev, lddn, op->h_dtype, true},         {dout_dev, lddout, op->r_dtype, false}, {r_dev, ldr, op->r_dtype, true},
      {h_dev, ldh, op->h_dtype, false},          {g.dr_dev, g.ld_dr, op->r_dtype, false}, {g.dh_dev, g.ld_dh, op->h_dtype, false}};
  for (const auto& x : arrays)
    if ((x.needed || x.p) && (rc = check_near_rows(x.p, x.ld, x.type, op->rows, op->d)) != SDS_OK) return rc;
  if (op->rows > 0 && !h_dev && (g.dh_dev || g.dgate_dev || g.dpost_w_dev)) return SDS_EINVAL;
  if (g.dpost_w_dev && !op->post) return SDS_EINVAL;
  for (const void* p : {(const void*)g.dw_dev, (const void*)g.db_dev, (const void*)g.dpost_w_dev})
    if (!aligned(p, type_bytes(op->w_dtype))) return SDS_EINVAL;
  if ((rc = check_cond(g.dgate_dev, g.ld_dgate, op->cond_dtype, op->groups, op->d)) != SDS_OK) return rc;
  if ((rc = check_cond(g.dscale_dev, g.ld_dscale, op->cond_dtype, op->groups, op->d)) != SDS_OK) return rc;
  if ((rc = check_cond(g.dshift_dev, g.ld_dshift, op->cond_dtype, op->groups, op->d)) != SDS_OK) return rc;
  if (op->rows > 0 && !keep_dev) return SDS_EINVAL;
  if (!aligned(keep_dev, kAlign)) return SDS_ENOMEM;
  if ((rc = check_workspace(workspace_dev, workspace_bytes, residual_norm_bytes(op))) != SDS_OK) return rc;
  if (!g.dr_dev && !g.dh_dev && !g.dw_dev && !g.db_dev && !g.dpost_w_dev && !g.dgate_dev && !g.dscale_dev && !g.dshift_dev) return SDS_OK;
  ResidualNormArgs a = residual_norm_args(op, r_dev, ldr, h_dev, ldh, keep_dev);
  a.dn = dn_dev; a.lddn = lddn;
  a.dr = dout_dev; a.lddr = lddout;
  a.dr_in = g.dr_dev; a.lddr_in = g.ld_dr;
  a.dh = g.dh_dev; a.lddh = g.ld_dh;
  a.dw = g.dw_dev; a.db = g.db_dev; a.dwp = g.dpost_w_dev;
  a.dgate = g.dgate_dev; a.dscale = g.dscale_dev; a.dshift = g.dshift_dev;
  a.lddgate = g.ld_dgate; a.lddscale = g.ld_dscale; a.lddshift = g.ld_dshift;
  if (op->rows > 0) {
    size_t part = 0, groups = 0;
    residual_norm_plan(&a, &part, &groups);
    a.part = static_cast<float*>(workspace_dev);
    a.group_part = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + align_up(part * 4));
  }
  return result(launch_residual_norm_backward(a, static_cast<cudaStream_t>(cuda_stream)));
}

#pragma GCC visibility pop
}  // extern "C"
