// Exported operators beside the layer solves: rows kept in 8 bits, LayerNorm on its own, gradients from kept rows, and what
// lies between logits and their gradient.
// Host code that checks arguments and enqueues; the kernels are in q8.hip, norm.hip, q8_grad.hip and logits.hip.
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
constexpr int32_t MOST_LOGITS = 1 << 24;
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
int check_logits(const mgrit_logits_desc* d) {
  if (!d || d->rows < 0 || d->cols < 1 || !known(d->dtype) || (d->id_dtype != MGRIT_IDS_I32 && d->id_dtype != MGRIT_IDS_I64)) return MGRIT_INVALID_ARG;
  if (!(d->temperature >= 1e-4f && d->temperature <= 1e4f)) return MGRIT_INVALID_ARG;
  return d->cols > MOST_LOGITS || d->rows > MOST_ROWS ? MGRIT_UNSUPPORTED : MGRIT_OK;
}
int check_top(const mgrit_logits_desc* d, int32_t top_k) {
  if (top_k < 0 || top_k > d->cols) return MGRIT_INVALID_ARG;
  return top_k > MGRIT_TOP_MOST ? MGRIT_UNSUPPORTED : MGRIT_OK;
}
int check_kept(int32_t kept) { return kept < 1 ? MGRIT_INVALID_ARG : kept > MGRIT_KEPT_MOST ? MGRIT_UNSUPPORTED : MGRIT_OK; }
int check_ids(const mgrit_logits_desc* d, const void* ids) {
  return d->rows == 0 || (ids && aligned(ids, d->id_dtype == MGRIT_IDS_I64 ? 8 : 4)) ? MGRIT_OK : MGRIT_INVALID_ARG;
}
int check_floats(const mgrit_logits_desc* d, const float* p) { return d->rows == 0 || (p && aligned(p, 4)) ? MGRIT_OK : MGRIT_INVALID_ARG; }
int check_teacher(const mgrit_logits_desc* d, const mgrit_teacher* t) {
  if (!t || !known(t->dtype)) return MGRIT_INVALID_ARG;
  STCHK(check_kept(t->kept));
  STCHK(check_ids(d, t->ids));
  return d->rows && (!t->logits || !element_aligned(t->logits, t->dtype) || !aligned(t->lse, 4)) ? MGRIT_INVALID_ARG : MGRIT_OK;
}
// What a call reads and writes: arrays of `row` bytes per row of logits, `stride` bytes apart.  While a result is written other blocks still
// read and write, so none lies on another or on an argument.  But a forward pass reads what it needs of a row before it writes the row's
// values: those may take the place of an argument, entry upon entry.  The logits' gradient against the logits: check_dlogits.
class Arrays {
  struct Span { const char* at; int64_t row, stride, rows; bool written; };
  Span all[16];
  int n = 0;
  int64_t rows;
  bool fine = true;
  static bool meet(const Span& a, const Span& b) {       // one of them without gaps between its rows
    const Span &s = a.row == a.stride ? b : a, &flat = a.row == a.stride ? a : b;
    const int64_t off = flat.at - s.at, bytes = flat.row * flat.rows;
    if (off >= (s.rows - 1) * s.stride + s.row || off + bytes <= 0) return false;
    return off < 0 || off % s.stride < s.row || off % s.stride + bytes > s.stride;
  }
  void add(const void* p, int64_t row, int64_t stride, int64_t count, bool written, bool upon) {
    if (!p || !row || !count) return;
    const Span s = {static_cast<const char*>(p), row, stride, count, written};
    for (int i = 0; written && i < n; ++i)
      fine = fine && (!meet(s, all[i]) || (upon && !all[i].written && all[i].at == s.at && all[i].row == row && all[i].stride == stride));
    all[n++] = s;
  }
 public:
  explicit Arrays(const mgrit_logits_desc* d) : rows(d->rows) {}
  Arrays& reads(const void* p, int64_t row) { add(p, row, row, rows, false, false); return *this; }
  Arrays& reads_rows(const void* p, int64_t row, int64_t stride) { add(p, row, stride, rows, false, false); return *this; }
  Arrays& writes(const void* p, int64_t row, bool upon = false) { add(p, row, row, rows, true, upon); return *this; }
  Arrays& writes_rows(const void* p, int64_t row, int64_t stride) { add(p, row, stride, rows, true, false); return *this; }     // (first of the results, logits after it)
  Arrays& writes_once(const void* p, int64_t bytes) { add(p, bytes, bytes, rows ? 1 : 0, true, false); return *this; }
  int check() const { return fine ? MGRIT_OK : MGRIT_INVALID_ARG; }
};
int64_t elem_bytes(int dtype) { return dtype == MGRIT_DTYPE_BF16 ? 2 : 4; }
int64_t id_bytes(const mgrit_logits_desc* d) { return d->id_dtype == MGRIT_IDS_I64 ? 8 : 4; }
Arrays& read_logits(Arrays& a, const mgrit_logits_desc* d, const void* logits, int64_t stride) {
  return a.reads_rows(logits, d->cols * elem_bytes(d->dtype), stride * elem_bytes(d->dtype));
}
Arrays& write_dlogits(Arrays& a, const mgrit_logits_desc* d, const void* dlogits, int64_t stride) {
  return a.writes_rows(dlogits, d->cols * elem_bytes(d->dtype), stride * elem_bytes(d->dtype));
}
Arrays& read_teacher(Arrays& a, const mgrit_logits_desc* d, const mgrit_teacher* t) {
  return a.reads(t->ids, t->kept * id_bytes(d)).reads(t->logits, t->kept * elem_bytes(t->dtype)).reads(t->lse, 4);
}
// gradients beside the logits, or in their place: nowhere across them
int check_dlogits(const mgrit_logits_desc* d, const void* logits, int64_t stride, const void* dlogits, int64_t dstride) {
  STCHK(check_rows(d->rows, d->cols, dlogits, dstride, d->dtype));
  if (d->rows == 0) return MGRIT_OK;
  const int64_t size = elem_bytes(d->dtype), apart = static_cast<const char*>(dlogits) - static_cast<const char*>(logits);
  const int64_t z_bytes = ((d->rows - 1) * stride + d->cols) * size, dz_bytes = ((d->rows - 1) * dstride + d->cols) * size;
  if (apart >= z_bytes || -apart >= dz_bytes) return MGRIT_OK;
  if (d->rows > 1 && stride != dstride) return MGRIT_INVALID_ARG;
  if (apart == 0) return MGRIT_OK;
  // slices of the same wider rows
  const int64_t at = (apart / size % stride + stride) % stride;
  return apart % size == 0 && d->rows > 1 && at >= d->cols && at <= stride - d->cols ? MGRIT_OK : MGRIT_INVALID_ARG;
}
LogitsArgs logits_args(const mgrit_logits_desc* d, const void* logits, int64_t stride) {
  LogitsArgs a = {};
  a.rows = d->rows; a.cols = d->cols; a.z = logits; a.ld = stride; a.tau = d->temperature; a.wide_ids = d->id_dtype == MGRIT_IDS_I64;
  return a;
}
void add_teacher(LogitsArgs& a, const mgrit_teacher* t) {
  a.kept = t->kept; a.teacher_ids = t->ids; a.teacher = t->logits; a.teacher_bf16 = t->dtype == MGRIT_DTYPE_BF16; a.teacher_lse = t->lse;
}
int enqueue_logits(const mgrit_logits_desc* d, const LogitsArgs& a, int mode, void* workspace, void* stream) {
  std::lock_guard<std::recursive_mutex> call_lock(call_mutex());
  return enqueued(launch_logits(a, mode, d->dtype == MGRIT_DTYPE_BF16, workspace, static_cast<hipStream_t>(stream)));
}
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

size_t mgrit_token_logprobs_workspace_bytes(const mgrit_logits_desc* desc, int32_t top_k, int step) {
  if (check_logits(desc) != MGRIT_OK || check_top(desc, top_k) != MGRIT_OK) return 0;
  return logits_workspace_bytes(desc->rows, desc->cols, desc->dtype == MGRIT_DTYPE_BF16, step ? 0 : top_k, 1, step != 0);
}

int mgrit_token_logprobs_forward(const mgrit_logits_desc* desc, const void* logits, int64_t stride, const void* tokens, float* logprob,
                                 float* entropy, float* lse, int32_t top_k, void* top_ids, float* top_logprobs, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  STCHK(check_logits(desc));
  STCHK(check_top(desc, top_k));
  STCHK(check_rows(desc->rows, desc->cols, logits, stride, desc->dtype));
  if (logprob || tokens) STCHK(check_ids(desc, tokens));
  if (desc->rows && !logprob && !entropy && !lse && !top_k) return MGRIT_INVALID_ARG;
  if (!aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(lse, 4)) return MGRIT_INVALID_ARG;
  if (top_k) {
    STCHK(check_ids(desc, top_ids));
    STCHK(check_floats(desc, top_logprobs));
  }
  const size_t need = mgrit_token_logprobs_workspace_bytes(desc, top_k, 0);
  STCHK(check_workspace(need, workspace, workspace_bytes));
  Arrays arrays(desc);
  read_logits(arrays, desc, logits, stride).reads(tokens, id_bytes(desc)).writes(logprob, 4, true).writes(entropy, 4, true).writes(lse, 4, true);
  arrays.writes(top_k ? top_ids : nullptr, top_k * id_bytes(desc)).writes(top_k ? top_logprobs : nullptr, top_k * 4, true);
  STCHK(arrays.writes_once(workspace, need).check());
  LogitsArgs a = logits_args(desc, logits, stride);
  a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.lse = lse; a.top_k = top_k; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  return enqueue_logits(desc, a, 0, workspace, stream);
}

int mgrit_token_logprobs_backward(const mgrit_logits_desc* desc, const void* logits, int64_t stride, const void* tokens, const float* lse,
                                  const float* g_logprob, const float* entropy, const float* g_entropy, void* dlogits,
                                  int64_t dlogits_stride, void* stream) {
  STCHK(check_logits(desc));
  STCHK(check_rows(desc->rows, desc->cols, logits, stride, desc->dtype));
  STCHK(check_ids(desc, tokens));
  STCHK(check_floats(desc, lse));
  STCHK(check_floats(desc, g_logprob));
  if (g_entropy) {
    STCHK(check_floats(desc, entropy));
    STCHK(check_floats(desc, g_entropy));
  }
  STCHK(check_dlogits(desc, logits, stride, dlogits, dlogits_stride));
  Arrays arrays(desc);
  arrays.reads(tokens, id_bytes(desc)).reads(lse, 4).reads(g_logprob, 4).reads(g_entropy ? entropy : nullptr, 4).reads(g_entropy, 4);
  STCHK(write_dlogits(arrays, desc, dlogits, dlogits_stride).check());
  LogitsArgs a = logits_args(desc, logits, stride);
  a.tokens = tokens; a.lse_in = lse; a.entropy_in = entropy; a.g = g_logprob; a.h = g_entropy; a.dz = dlogits; a.lddz = dlogits_stride;
  return enqueue_logits(desc, a, 0, nullptr, stream);
}

int mgrit_token_logprobs_step(const mgrit_logits_desc* desc, const void* logits, int64_t stride, const void* tokens, const float* g_logprob,
                              const float* g_entropy, float* logprob, float* entropy, float* lse, void* dlogits, int64_t dlogits_stride,
                              void* workspace, size_t workspace_bytes, void* stream) {
  STCHK(check_logits(desc));
  STCHK(check_rows(desc->rows, desc->cols, logits, stride, desc->dtype));
  STCHK(check_ids(desc, tokens));
  STCHK(check_floats(desc, g_logprob));
  if (!aligned(g_entropy, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(lse, 4)) return MGRIT_INVALID_ARG;
  STCHK(check_dlogits(desc, logits, stride, dlogits, dlogits_stride));
  const size_t need = mgrit_token_logprobs_workspace_bytes(desc, 0, 1);
  STCHK(check_workspace(need, workspace, workspace_bytes));
  Arrays arrays(desc);
  arrays.reads(tokens, id_bytes(desc)).reads(g_logprob, 4).reads(g_entropy, 4);
  read_logits(write_dlogits(arrays, desc, dlogits, dlogits_stride), desc, logits, stride).writes(logprob, 4).writes(entropy, 4).writes(lse, 4);
  STCHK(arrays.writes_once(workspace, need).check());
  LogitsArgs a = logits_args(desc, logits, stride);
  a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.lse = lse; a.g = g_logprob; a.h = g_entropy; a.dz = dlogits; a.lddz = dlogits_stride;
  return enqueue_logits(desc, a, 0, workspace, stream);
}

size_t mgrit_distill_workspace_bytes(const mgrit_logits_desc* desc, int32_t kept, int step) {
  if (check_logits(desc) != MGRIT_OK || check_kept(kept) != MGRIT_OK) return 0;
  return logits_workspace_bytes(desc->rows, desc->cols, desc->dtype == MGRIT_DTYPE_BF16, 0, kept, step != 0);
}

int mgrit_distill_forward(const mgrit_logits_desc* desc, const void* logits, int64_t stride, const mgrit_teacher* teacher, float* loss,
                          float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  STCHK(check_logits(desc));
  STCHK(check_rows(desc->rows, desc->cols, logits, stride, desc->dtype));
  STCHK(check_teacher(desc, teacher));
  STCHK(check_floats(desc, loss));
  if (!aligned(lse, 4)) return MGRIT_INVALID_ARG;
  const size_t need = mgrit_distill_workspace_bytes(desc, teacher->kept, 0);
  STCHK(check_workspace(need, workspace, workspace_bytes));
  Arrays arrays(desc);
  read_teacher(read_logits(arrays, desc, logits, stride), desc, teacher).writes(loss, 4, true).writes(lse, 4, true);
  STCHK(arrays.writes_once(workspace, need).check());
  LogitsArgs a = logits_args(desc, logits, stride);
  add_teacher(a, teacher);
  a.loss = loss; a.lse = lse;
  return enqueue_logits(desc, a, 1, workspace, stream);
}

int mgrit_distill_backward(const mgrit_logits_desc* desc, const void* logits, int64_t stride, const mgrit_teacher* teacher, const float* lse,
                           const float* g_loss, void* dlogits, int64_t dlogits_stride, void* stream) {
  STCHK(check_logits(desc));
  STCHK(check_rows(desc->rows, desc->cols, logits, stride, desc->dtype));
  STCHK(check_teacher(desc, teacher));
  STCHK(check_floats(desc, lse));
  if (!aligned(g_loss, 4)) return MGRIT_INVALID_ARG;
  STCHK(check_dlogits(desc, logits, stride, dlogits, dlogits_stride));
  Arrays arrays(desc);
  read_teacher(arrays, desc, teacher).reads(lse, 4).reads(g_loss, 4);
  STCHK(write_dlogits(arrays, desc, dlogits, dlogits_stride).check());
  LogitsArgs a = logits_args(desc, logits, stride);
  add_teacher(a, teacher);
  a.lse_in = lse; a.g = g_loss; a.dz = dlogits; a.lddz = dlogits_stride;
  return enqueue_logits(desc, a, 1, nullptr, stream);
}

int mgrit_distill_step(const mgrit_logits_desc* desc, const void* logits, int64_t stride, const mgrit_teacher* teacher, const float* g_loss,
                       float* loss, float* lse, void* dlogits, int64_t dlogits_stride, void* workspace, size_t workspace_bytes, void* stream) {
  STCHK(check_logits(desc));
  STCHK(check_rows(desc->rows, desc->cols, logits, stride, desc->dtype));
  STCHK(check_teacher(desc, teacher));
  STCHK(check_floats(desc, loss));
  if (!aligned(g_loss, 4) || !aligned(lse, 4)) return MGRIT_INVALID_ARG;
  STCHK(check_dlogits(desc, logits, stride, dlogits, dlogits_stride));
  const size_t need = mgrit_distill_workspace_bytes(desc, teacher->kept, 1);
  STCHK(check_workspace(need, workspace, workspace_bytes));
  Arrays arrays(desc);
  read_teacher(arrays, desc, teacher).reads(g_loss, 4);
  read_logits(write_dlogits(arrays, desc, dlogits, dlogits_stride), desc, logits, stride).writes(loss, 4).writes(lse, 4);
  STCHK(arrays.writes_once(workspace, need).check());
  LogitsArgs a = logits_args(desc, logits, stride);
  add_teacher(a, teacher);
  a.loss = loss; a.lse = lse; a.g = g_loss; a.dz = dlogits; a.lddz = dlogits_stride;
  return enqueue_logits(desc, a, 1, workspace, stream);
}

}  // extern "C"
