// Exported operators beside the layer solves: rows kept in 8 bits, LayerNorm on its own, gradients from kept rows.
// Host code that checks arguments and enqueues; the kernels are in q8.hip, norm.hip and q8_grad.hip.
#include <math.h>

#include "../../include/mgrit.h"
#include "api.h"
#include "kernels.h"
#include "q8.h"

using namespace mg;

namespace {

#define STCHK(expr)                                    \
  do {                                                 \
    int s_ = (expr);                                   \
    if (s_ != MGRIT_OK) return s_;                     \
  } while (0)

constexpr int64_t MOST_ROWS = 0x7fffffff;
constexpr int32_t MOST_NORM_COLS = 16384;              // a row lies in the registers of 1024 lanes
constexpr int64_t MOST_ELEMENTS = (int64_t)1 << 40, MOST_WEIGHTS = (int64_t)1 << 31;
constexpr int32_t MOST_FEATURES = 1 << 24;
constexpr int64_t MOST_TOKENS = MOST_ROWS - 255;       // the index of a token behind the last one, in its tile, has 32 bits

bool known(int dtype) { return dtype == MGRIT_DTYPE_F32 || dtype == MGRIT_DTYPE_BF16; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool element_aligned(const void* p, int dtype) { return aligned(p, dtype == MGRIT_DTYPE_BF16 ? 2 : 4); }

// a matrix argument: present if there are rows, rows no closer than they are long
int check_rows(int64_t rows, int64_t cols, const void* p, int64_t stride, int dtype) {
  if (rows == 0) return MGRIT_OK;
  if (!p || !element_aligned(p, dtype) || stride < cols) return MGRIT_INVALID_ARG;
  return stride > MOST_ELEMENTS / rows ? MGRIT_UNSUPPORTED : MGRIT_OK;
}
int check_q8(int64_t rows, const void* q, const void* scale) {
  return rows == 0 || (q && scale && aligned(q, 16)) ? MGRIT_OK : MGRIT_INVALID_ARG;
}
int check_q8_shape(int64_t rows, int32_t cols) {
  if (rows < 0 || cols < 1) return MGRIT_INVALID_ARG;
  return rows > MOST_ELEMENTS / cols ? MGRIT_UNSUPPORTED : MGRIT_OK;
}
int check_norm(const mgrit_norm_desc* d) {
  if (!d || d->rows < 0 || d->cols < 1 || !known(d->x_dtype) || !known(d->y_dtype)) return MGRIT_INVALID_ARG;
  if (!(d->eps > 0.f) || !isfinite(d->eps)) return MGRIT_INVALID_ARG;
  return d->cols > MOST_NORM_COLS || d->rows > MOST_ROWS ? MGRIT_UNSUPPORTED : MGRIT_OK;
}
// the optional 8-bit copy of a row matrix: both arrays or none
int check_copy(const void* q, const void* scale) {
  return (!q && !scale) || (q && scale && aligned(q, 16)) ? MGRIT_OK : MGRIT_INVALID_ARG;
}
int check_weight_grad(int64_t rows, int32_t out_features, int32_t in_features, int dy_dtype) {
  if (rows < 0 || out_features < 1 || in_features < 1 || !known(dy_dtype)) return MGRIT_INVALID_ARG;
  if (out_features > MOST_FEATURES || in_features > MOST_FEATURES) return MGRIT_UNSUPPORTED;
  return rows > MOST_TOKENS || (int64_t)out_features * in_features > MOST_WEIGHTS ? MGRIT_UNSUPPORTED : MGRIT_OK;
}
int check_workspace(size_t need, const void* workspace, size_t bytes) {
  if (!need) return MGRIT_OK;
  if (!workspace || !aligned(workspace, 256)) return MGRIT_INVALID_ARG;
  return bytes < need ? MGRIT_WORKSPACE_TOO_SMALL : MGRIT_OK;
}
int enqueued(hipError_t e) { return e == hipSuccess ? MGRIT_OK : hip_failed(e); }
Q8Rows kept(int64_t rows, int32_t cols, const void* q, const void* scale) {
  return Q8Rows{static_cast<unsigned char*>(const_cast<void*>(q)), static_cast<unsigned char*>(const_cast<void*>(scale)), rows, cols};
}

}  // namespace

extern "C" {

int64_t mgrit_q8_blocks(int32_t cols) { return cols < 1 ? 0 : q8_blocks(cols); }

int mgrit_q8_pack(int64_t rows, int32_t cols, int dtype, const void* x, int64_t x_stride, void* q, void* scale, void* stream) {
  if (!known(dtype)) return MGRIT_INVALID_ARG;
  STCHK(check_q8_shape(rows, cols));
  STCHK(check_rows(rows, cols, x, x_stride, dtype));
  STCHK(check_q8(rows, q, scale));
  std::lock_guard<std::recursive_mutex> call_lock(call_mutex());
  return enqueued(launch_q8_pack(kept(rows, cols, q, scale), x, x_stride, dtype == MGRIT_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

int mgrit_q8_unpack(int64_t rows, int32_t cols, int dtype, const void* q, const void* scale, void* x, int64_t x_stride, void* stream) {
  if (!known(dtype)) return MGRIT_INVALID_ARG;
  STCHK(check_q8_shape(rows, cols));
  STCHK(check_rows(rows, cols, x, x_stride, dtype));
  STCHK(check_q8(rows, q, scale));
  std::lock_guard<std::recursive_mutex> call_lock(call_mutex());
  return enqueued(launch_q8_unpack(kept(rows, cols, q, scale), x, x_stride, dtype == MGRIT_DTYPE_BF16, 1, 0, 0, static_cast<hipStream_t>(stream)));
}

int mgrit_layer_norm_forward(const mgrit_norm_desc* desc, const void* x, int64_t x_stride, const float* gamma,
                             const float* beta, void* y, int64_t y_stride, float* mean, float* rstd, void* x_q8,
                             void* x_q8_scale, void* y_q8, void* y_q8_scale, void* stream) {
  STCHK(check_norm(desc));
  STCHK(check_rows(desc->rows, desc->cols, x, x_stride, desc->x_dtype));
  STCHK(check_rows(desc->rows, desc->cols, y, y_stride, desc->y_dtype));
  if (!aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return MGRIT_INVALID_ARG;
  STCHK(check_copy(x_q8, x_q8_scale));
  STCHK(check_copy(y_q8, y_q8_scale));
  if ((y_q8 && (y_q8 == x_q8 || y_q8_scale == x_q8_scale)) || (mean && mean == rstd)) return MGRIT_INVALID_ARG;
  // in place: every row is read before it is written, if it keeps its place
  if (desc->rows && x == y && (x_stride != y_stride || desc->x_dtype != desc->y_dtype)) return MGRIT_INVALID_ARG;
  std::lock_guard<std::recursive_mutex> call_lock(call_mutex());
  NormFwdArgs a = {};
  a.rows = desc->rows; a.cols = desc->cols; a.blocks = (int)q8_blocks(desc->cols); a.eps = desc->eps;
  a.x = x; a.ldx = x_stride; a.gamma = gamma; a.beta = beta;
  a.y = y; a.ldy = y_stride; a.y_bf16 = desc->y_dtype == MGRIT_DTYPE_BF16; a.mean = mean; a.rstd = rstd;
  a.xq = static_cast<unsigned char*>(x_q8); a.xs = static_cast<unsigned char*>(x_q8_scale);
  a.yq = static_cast<unsigned char*>(y_q8); a.ys = static_cast<unsigned char*>(y_q8_scale);
  return enqueued(launch_norm_forward(a, desc->x_dtype == MGRIT_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

size_t mgrit_layer_norm_backward_workspace_bytes(const mgrit_norm_desc* desc) {
  return check_norm(desc) == MGRIT_OK ? 4 * norm_backward_partial_floats(desc->rows, desc->cols) : 0;
}

int mgrit_layer_norm_backward(const mgrit_norm_desc* desc, const void* dy, int64_t dy_stride, const void* x,
                              int64_t x_stride, const void* x_q8, const void* x_q8_scale, const float* gamma,
                              const float* mean, const float* rstd, void* dx, int64_t dx_stride, float* dgamma,
                              float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
  STCHK(check_norm(desc));
  if ((x != nullptr) == (x_q8 != nullptr) && desc->rows) return MGRIT_INVALID_ARG;       // one of the two
  if (!dx && !dgamma && !dbeta) return MGRIT_INVALID_ARG;
  STCHK(check_rows(desc->rows, desc->cols, dy, dy_stride, desc->y_dtype));
  if (x) STCHK(check_rows(desc->rows, desc->cols, x, x_stride, desc->x_dtype));
  STCHK(check_copy(x_q8, x_q8_scale));
  if (dx) STCHK(check_rows(desc->rows, desc->cols, dx, dx_stride, desc->x_dtype));
  if (desc->rows && (!mean || !rstd)) return MGRIT_INVALID_ARG;
  if (!aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4)) return MGRIT_INVALID_ARG;
  if ((dx && (dx == dy || dx == x)) || (dgamma && dgamma == dbeta)) return MGRIT_INVALID_ARG;
  if (dgamma || dbeta) STCHK(check_workspace(mgrit_layer_norm_backward_workspace_bytes(desc), workspace, workspace_bytes));
  std::lock_guard<std::recursive_mutex> call_lock(call_mutex());
  NormBwdArgs a = {};
  a.rows = desc->rows; a.cols = desc->cols; a.blocks = (int)q8_blocks(desc->cols);
  a.dy = dy; a.ldy = dy_stride; a.x = x; a.ldx = x_stride; a.x_bf16 = desc->x_dtype == MGRIT_DTYPE_BF16;
  a.xq = static_cast<const unsigned char*>(x_q8); a.xs = static_cast<const unsigned char*>(x_q8_scale);
  a.gamma = gamma; a.mean = mean; a.rstd = rstd; a.dx = dx; a.lddx = dx_stride; a.dgamma = dgamma; a.dbeta = dbeta;
  return enqueued(launch_norm_backward(a, desc->y_dtype == MGRIT_DTYPE_BF16, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

size_t mgrit_q8_weight_grad_workspace_bytes(int64_t rows, int32_t out_features, int32_t in_features, int dy_dtype) {
  if (check_weight_grad(rows, out_features, in_features, dy_dtype) != MGRIT_OK) return 0;
  return 4 * q8_grad_partial_floats(rows, out_features, in_features, dy_dtype == MGRIT_DTYPE_BF16);
}

int mgrit_q8_weight_grad(int64_t rows, int32_t out_features, int32_t in_features, int dy_dtype, const void* dy,
                         int64_t dy_stride, const void* x_q8, const void* x_q8_scale, float scale, float* dW, float* db,
                         void* workspace, size_t workspace_bytes, void* stream) {
  STCHK(check_weight_grad(rows, out_features, in_features, dy_dtype));
  STCHK(check_rows(rows, out_features, dy, dy_stride, dy_dtype));
  if (rows && dy_stride > MOST_FEATURES) return MGRIT_UNSUPPORTED;        // a tile's offsets have 32 bits
  STCHK(check_q8(rows, x_q8, x_q8_scale));
  if (!dW || !aligned(dW, 4) || !aligned(db, 4) || dW == db || !isfinite(scale)) return MGRIT_INVALID_ARG;
  STCHK(check_workspace(mgrit_q8_weight_grad_workspace_bytes(rows, out_features, in_features, dy_dtype), workspace, workspace_bytes));
  std::lock_guard<std::recursive_mutex> call_lock(call_mutex());
  Q8GradArgs a = {};
  a.rows = rows; a.M = out_features; a.N = in_features; a.dy = dy; a.ldy = dy_stride;
  a.xq = static_cast<const unsigned char*>(x_q8); a.xs = static_cast<const unsigned char*>(x_q8_scale);
  a.blocks = (int)q8_blocks(in_features); a.dW = dW; a.db = db; a.scale = scale;
  return enqueued(launch_q8_grad(a, dy_dtype == MGRIT_DTYPE_BF16, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
