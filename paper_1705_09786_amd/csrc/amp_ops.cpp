// C entry points of the operators on whole arrays (include/amp.h): argument checks and launches.  Nothing here allocates, waits or
// throws.
#include <stdarg.h>
#include <stdio.h>

#include "../../include/amp.h"
#include "amp_ops.h"

namespace {

thread_local char g_error[256] = "no error";

__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_error, sizeof g_error, fmt, ap);
  va_end(ap);
  return code;
}

// An earlier asynchronous error of the device is left for whoever waits for it; only the launch's own status counts here.
int launched(const char* what, hipError_t e) {
  return e == hipSuccess ? AMP_OK : fail(AMP_EDEVICE, "%s: launch failed: %s", what, hipGetErrorString(e));
}

constexpr size_t MAX_ROWS = (size_t)1 << 31, MAX_COLS = (size_t)1 << 31, MAX_EXTENT = (size_t)1 << 56;

size_t elem(int dtype) { return dtype == AMP_F32 ? 4 : 2; }

int check_size(const char* what, int dtype, size_t rows, size_t cols, const char* cols_name) {
  if (dtype < AMP_F32 || dtype > AMP_F16) return fail(AMP_EINVAL, "%s: unknown dtype %d", what, dtype);
  if (rows >= MAX_ROWS) return fail(AMP_EINVAL, "%s: %zu rows, fewer than 2^31 are taken", what, rows);
  if (cols < 1 || cols >= MAX_COLS) return fail(AMP_EINVAL, "%s: %s = %zu, 1 .. 2^31 - 1 are taken", what, cols_name, cols);
  return AMP_OK;
}

// A 2-D array as far as overlaps go: rows of `cols` elements of `size` bytes, `stride` elements apart.
struct Span {
  const char* name;
  const void* p;
  size_t rows, cols, stride, size;
  uintptr_t first() const { return (uintptr_t)p; }
  uintptr_t last() const { return first() + ((rows - 1) * stride + cols) * size; }   // one past it
};

bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || !a.rows || !b.rows || !a.cols || !b.cols) return false;
  if (a.last() <= b.first() || b.last() <= a.first()) return false;
  const size_t step = a.stride * a.size;
  if (step != b.stride * b.size || a.rows == 1 || b.rows == 1 || step == 0) return true;
  // the same row distance: apart where their columns are apart in every row, counted round the row
  const size_t wa = a.cols * a.size, wb = b.cols * b.size;
  const size_t d = (b.first() >= a.first() ? b.first() - a.first() : step - (a.first() - b.first()) % step) % step;
  return d < wa || step - d < wb;
}

int check_array(const char* what, const Span& s, bool output) {
  if (s.rows == 0) return AMP_OK;
  if (!s.p) return fail(AMP_EINVAL, "%s: %s is NULL", what, s.name);
  if (s.first() % s.size) return fail(AMP_EINVAL, "%s: %s is not aligned to its %zu-byte elements", what, s.name, s.size);
  if (s.stride > MAX_EXTENT / s.rows || s.cols > MAX_EXTENT / s.rows)
    return fail(AMP_EINVAL, "%s: %s spans 2^56 elements or more", what, s.name);
  if (output && s.rows > 1 && s.stride < s.cols)
    return fail(AMP_EINVAL, "%s: rows of %s overlap: stride %zu, row %zu", what, s.name, s.stride, s.cols);
  return AMP_OK;
}

bool same(const Span& a, const Span& b) { return a.p == b.p && a.size == b.size && (a.rows <= 1 || a.stride == b.stride); }

// The first n_out of the arrays are outputs.  pair[i] (if any) is the array that output i may also be.
template <int N>
int check_overlaps(const char* what, const Span (&s)[N], int n_out, const int (*pair)[2], int n_pairs) {
  for (int i = 0; i < n_out; ++i)
    for (int j = i + 1; j < N; ++j) {
      if (!overlap(s[i], s[j])) continue;
      bool allowed = false;
      for (int k = 0; k < n_pairs; ++k) allowed = allowed || (pair[k][0] == i && pair[k][1] == j && same(s[i], s[j]));
      if (!allowed) return fail(AMP_EINVAL, "%s: %s overlaps %s", what, s[i].name, s[j].name);
    }
  return AMP_OK;
}

int check_workspace(const char* what, const void* ws, size_t have, size_t need) {
  if (need == 0) return AMP_OK;
  if (!ws) return fail(AMP_EINVAL, "%s: workspace is NULL, %zu bytes are needed", what, need);
  if ((uintptr_t)ws & 15) return fail(AMP_EINVAL, "%s: workspace is not 16-byte aligned", what);
  if (have < need) return fail(AMP_ENOMEM, "%s: workspace of %zu bytes, %zu are needed", what, have, need);
  return AMP_OK;
}

#define CHECK(call)                 \
  do {                              \
    const int rc_ = (call);         \
    if (rc_ != AMP_OK) return rc_;  \
  } while (0)

template <int N>
int check_arrays(const char* what, const Span (&s)[N], int n_out) {
  for (int i = 0; i < N; ++i)
    if (s[i].p) CHECK(check_array(what, s[i], i < n_out));
  return AMP_OK;
}

int check_scan_size(const char* what, int dtype, size_t rows, size_t hidden) {
  CHECK(check_size(what, dtype, rows, hidden, "hidden"));
  if (rows >= MAX_ROWS / 2) return fail(AMP_EINVAL, "%s: %zu rows, fewer than 2^30 are taken", what, rows);
  if (hidden >= (size_t)1 << 22) return fail(AMP_EINVAL, "%s: hidden = %zu, 1 .. 2^22 - 1 are taken", what, hidden);
  // a launch has fewer than 2^24 workgroups of 256 threads, each of them 128 rows by 64 features
  if (rows > ((size_t)1 << 36) / hidden) return fail(AMP_EINVAL, "%s: %zu rows of %zu, up to 2^36 elements are taken", what, rows, hidden);
  return AMP_OK;
}

// The scan's kernels reach a tile's rows by 32-bit offsets.
int check_scan_stride(const char* what, const char* name, size_t stride) {
  return stride < (size_t)1 << 22 ? AMP_OK : fail(AMP_EINVAL, "%s: %s has a row stride of 2^22 or more", what, name);
}

int check_scan(const char* what, int dtype, int activation, size_t rows, size_t hidden, const amp_sequences* q) {
  CHECK(check_scan_size(what, dtype, rows, hidden));
  if (activation != AMP_ACT_NONE && activation != AMP_ACT_TANH)
    return fail(AMP_EINVAL, "%s: activation %d, AMP_ACT_NONE and AMP_ACT_TANH are taken", what, activation);
  if (!q) return fail(AMP_EINVAL, "%s: sequences is NULL", what);
  if (q->n >= MAX_ROWS) return fail(AMP_EINVAL, "%s: %zu sequences, fewer than 2^31 are taken", what, q->n);
  if (q->zero_others != 0 && q->zero_others != 1) return fail(AMP_EINVAL, "%s: zero_others %d, 0 and 1 are taken", what, q->zero_others);
  if (!q->begin != !q->end) return fail(AMP_EINVAL, "%s: one of begin and end is NULL", what);
  if (!q->begin) {
    if (q->n > 1) return fail(AMP_EINVAL, "%s: %zu sequences without begin and end", what, q->n);
    return AMP_OK;
  }
  if (q->index_bytes != 4 && q->index_bytes != 8) return fail(AMP_EINVAL, "%s: index_bytes %d, 4 and 8 are taken", what, q->index_bytes);
  if ((uintptr_t)q->begin % q->index_bytes || (uintptr_t)q->end % q->index_bytes)
    return fail(AMP_EINVAL, "%s: begin or end is not aligned to its elements", what);
  return AMP_OK;
}

#define REQUIRE(p)                                                              \
  do {                                                                          \
    if (!(p)) return fail(AMP_EINVAL, "%s: %s is NULL", what, #p);              \
  } while (0)

}  // namespace

extern "C" {

const char* amp_operator_error(void) { return g_error; }

int amp_layer_norm_forward(int dtype, size_t rows, size_t cols, const void* x, size_t x_stride, const float* weight, const float* bias,
                           float eps, void* y, size_t y_stride, float* mean, float* rstd, void* hip_stream) {
  const char* what = "layer_norm_forward";
  CHECK(check_size(what, dtype, rows, cols, "cols"));
  if (!(eps >= 0.f)) return fail(AMP_EINVAL, "%s: eps is negative or not a number", what);
  if (rows == 0) return AMP_OK;
  REQUIRE(x);
  REQUIRE(y);
  const size_t e = elem(dtype);
  const Span s[] = {{"y", y, rows, cols, y_stride, e},   {"mean", mean, 1, rows, rows, 4},  {"rstd", rstd, 1, rows, rows, 4},
                    {"x", x, rows, cols, x_stride, e},   {"weight", weight, 1, cols, cols, 4}, {"bias", bias, 1, cols, cols, 4}};
  CHECK(check_arrays(what, s, 3));
  const int pair[][2] = {{0, 3}};
  CHECK(check_overlaps(what, s, 3, pair, 1));
  NormArgs a = {};
  a.rows = rows, a.cols = cols, a.x = x, a.x_stride = x_stride, a.weight = weight, a.bias = bias, a.eps = eps;
  a.y = y, a.y_stride = y_stride, a.mean = mean, a.rstd = rstd;
  return launched(what, amp_norm_forward_launch(dtype, &a, (hipStream_t)hip_stream));
}

int amp_layer_norm_workspace(int dtype, size_t rows, size_t cols, size_t* bytes) {
  const char* what = "layer_norm_workspace";
  CHECK(check_size(what, dtype, rows, cols, "cols"));
  REQUIRE(bytes);
  *bytes = amp_norm_workspace_bytes(dtype, rows, cols);
  return AMP_OK;
}

int amp_layer_norm_backward(int dtype, size_t rows, size_t cols, const void* dy, size_t dy_stride, const void* x, size_t x_stride,
                            const float* weight, const float* mean, const float* rstd, void* dx, size_t dx_stride, float* dweight,
                            float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* what = "layer_norm_backward";
  CHECK(check_size(what, dtype, rows, cols, "cols"));
  const size_t e = elem(dtype), need = dweight || dbias ? amp_norm_workspace_bytes(dtype, rows, cols) : 0;
  if (rows) {
    REQUIRE(x);
    REQUIRE(dy);
    REQUIRE(mean);
    REQUIRE(rstd);
  }
  const Span s[] = {{"dx", dx, rows, cols, dx_stride, e},       {"dweight", dweight, 1, cols, cols, 4}, {"dbias", dbias, 1, cols, cols, 4},
                    {"workspace", need ? workspace : nullptr, 1, need, need, 1},
                    {"dy", dy, rows, cols, dy_stride, e},       {"x", x, rows, cols, x_stride, e},      {"weight", weight, 1, cols, cols, 4},
                    {"mean", mean, 1, rows, rows, 4},           {"rstd", rstd, 1, rows, rows, 4}};
  CHECK(check_arrays(what, s, 4));
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  const int pair[][2] = {{0, 4}, {0, 5}};
  CHECK(check_overlaps(what, s, 4, pair, 2));
  if (!dx && !dweight && !dbias) return AMP_OK;
  NormArgs a = {};
  a.rows = rows, a.cols = cols, a.x = x, a.x_stride = x_stride, a.dy = dy, a.dy_stride = dy_stride, a.weight = weight;
  a.mean = (float*)mean, a.rstd = (float*)rstd, a.dx = dx, a.dx_stride = dx_stride, a.dweight = dweight, a.dbias = dbias;
  a.workspace = (float*)workspace;
  return launched(what, amp_norm_backward_launch(dtype, &a, (hipStream_t)hip_stream));
}

int amp_gated_scan_carry(int dtype, size_t rows, size_t hidden, size_t* carry_rows) {
  const char* what = "gated_scan_carry";
  CHECK(check_scan_size(what, dtype, rows, hidden));
  REQUIRE(carry_rows);
  *carry_rows = amp_scan_carry_rows(dtype, rows, hidden);
  return AMP_OK;
}

int amp_gated_scan_workspace(int dtype, size_t rows, size_t hidden, size_t* bytes) {
  const char* what = "gated_scan_workspace";
  CHECK(check_scan_size(what, dtype, rows, hidden));
  REQUIRE(bytes);
  *bytes = amp_scan_workspace_bytes(dtype, rows, hidden);
  return AMP_OK;
}

int amp_gated_scan_forward(int dtype, int activation, size_t rows, size_t hidden, const void* gate, size_t gate_stride, const void* cand,
                           size_t cand_stride, const amp_sequences* q, const float* h0, void* h, size_t h_stride, float* last,
                           float* carry, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* what = "gated_scan_forward";
  CHECK(check_scan(what, dtype, activation, rows, hidden, q));
  if ((q->n == 0 && !q->zero_others) || (!h && !last && !carry)) return AMP_OK;
  if (rows) {
    REQUIRE(gate);
    REQUIRE(cand);
  }
  const size_t e = elem(dtype), need = amp_scan_workspace_bytes(dtype, rows, hidden), n = q->n;
  const size_t nc = amp_scan_carry_rows(dtype, rows, hidden), ib = q->index_bytes;
  const Span s[] = {{"h", h, rows, hidden, h_stride, e},          {"last", last, n, hidden, hidden, 4},
                    {"carry", carry, nc, hidden, hidden, 4},      {"workspace", need ? workspace : nullptr, 1, need, need, 1},
                    {"gate", gate, rows, hidden, gate_stride, e}, {"cand", cand, rows, hidden, cand_stride, e},
                    {"h0", h0, n, hidden, hidden, 4},             {"begin", q->begin, 1, n, n, q->begin ? ib : 1},
                    {"end", q->end, 1, n, n, q->end ? ib : 1}};
  CHECK(check_arrays(what, s, 4));
  CHECK(check_scan_stride(what, "gate", gate_stride));
  CHECK(check_scan_stride(what, "cand", cand_stride));
  CHECK(check_scan_stride(what, "h", h_stride));
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  CHECK(check_overlaps(what, s, 4, nullptr, 0));
  ScanArgs a = {};
  a.rows = rows, a.hidden = hidden, a.gate = gate, a.gate_stride = gate_stride, a.cand = cand, a.cand_stride = cand_stride;
  a.n_seq = n, a.begin = q->begin, a.end = q->end, a.index_bytes = q->index_bytes, a.h0 = h0, a.h = h, a.h_stride = h_stride;
  a.zero_others = q->zero_others;
  a.last = last, a.carry = carry, a.workspace = workspace;
  return launched(what, amp_scan_forward_launch(dtype, activation == AMP_ACT_TANH, &a, (hipStream_t)hip_stream));
}

int amp_gated_scan_backward(int dtype, int activation, size_t rows, size_t hidden, const void* dh, size_t dh_stride, const float* dlast,
                            const void* gate, size_t gate_stride, const void* cand, size_t cand_stride, const amp_sequences* q,
                            const float* h0, const float* carry, void* dgate, size_t dgate_stride, void* dcand, size_t dcand_stride,
                            float* dh0, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* what = "gated_scan_backward";
  CHECK(check_scan(what, dtype, activation, rows, hidden, q));
  if (q->n == 0 && !q->zero_others) return AMP_OK;
  REQUIRE(carry);   // which has a row where there are no others
  if (rows) {
    REQUIRE(dh);
    REQUIRE(gate);
    REQUIRE(cand);
    REQUIRE(dgate);
    REQUIRE(dcand);
  }
  const size_t e = elem(dtype), need = amp_scan_workspace_bytes(dtype, rows, hidden), n = q->n;
  const size_t nc = amp_scan_carry_rows(dtype, rows, hidden), ib = q->index_bytes;
  const Span s[] = {{"dgate", dgate, rows, hidden, dgate_stride, e}, {"dcand", dcand, rows, hidden, dcand_stride, e},
                    {"dh0", dh0, n, hidden, hidden, 4},              {"workspace", need ? workspace : nullptr, 1, need, need, 1},
                    {"dh", dh, rows, hidden, dh_stride, e},          {"dlast", dlast, n, hidden, hidden, 4},
                    {"gate", gate, rows, hidden, gate_stride, e},    {"cand", cand, rows, hidden, cand_stride, e},
                    {"h0", h0, n, hidden, hidden, 4},                {"carry", carry, nc, hidden, hidden, 4},
                    {"begin", q->begin, 1, n, n, q->begin ? ib : 1}, {"end", q->end, 1, n, n, q->end ? ib : 1}};
  CHECK(check_arrays(what, s, 4));
  CHECK(check_scan_stride(what, "dh", dh_stride));
  CHECK(check_scan_stride(what, "gate", gate_stride));
  CHECK(check_scan_stride(what, "cand", cand_stride));
  CHECK(check_scan_stride(what, "dgate", dgate_stride));
  CHECK(check_scan_stride(what, "dcand", dcand_stride));
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  CHECK(check_overlaps(what, s, 4, nullptr, 0));
  ScanArgs a = {};
  a.rows = rows, a.hidden = hidden, a.dh = dh, a.dh_stride = dh_stride, a.dlast = dlast, a.gate = gate, a.gate_stride = gate_stride;
  a.cand = cand, a.cand_stride = cand_stride, a.n_seq = n, a.begin = q->begin, a.end = q->end, a.index_bytes = q->index_bytes;
  a.zero_others = q->zero_others, a.h0 = h0, a.carry_in = carry, a.dgate = dgate, a.dgate_stride = dgate_stride, a.dcand = dcand, a.dcand_stride = dcand_stride;
  a.dh0 = dh0, a.workspace = workspace;
  return launched(what, amp_scan_backward_launch(dtype, activation == AMP_ACT_TANH, &a, (hipStream_t)hip_stream));
}

int amp_gated_scan_step(int dtype, int activation, size_t rows, size_t hidden, const void* gate, size_t gate_stride, const void* cand,
                        size_t cand_stride, float* state, size_t state_stride, void* h, size_t h_stride, void* hip_stream) {
  const char* what = "gated_scan_step";
  const amp_sequences one = {1, nullptr, nullptr, 0, 0};
  CHECK(check_scan(what, dtype, activation, rows, hidden, &one));
  if (rows == 0) return AMP_OK;
  REQUIRE(gate);
  REQUIRE(cand);
  REQUIRE(state);
  const size_t e = elem(dtype);
  const Span s[] = {{"state", state, rows, hidden, state_stride, 4}, {"h", h, rows, hidden, h_stride, e},
                    {"gate", gate, rows, hidden, gate_stride, e},    {"cand", cand, rows, hidden, cand_stride, e}};
  CHECK(check_arrays(what, s, 2));
  CHECK(check_overlaps(what, s, 2, nullptr, 0));
  ScanStepArgs a = {};
  a.rows = rows, a.hidden = hidden, a.gate = gate, a.gate_stride = gate_stride, a.cand = cand, a.cand_stride = cand_stride;
  a.state = state, a.state_stride = state_stride, a.h = h, a.h_stride = h_stride;
  return launched(what, amp_scan_step_launch(dtype, activation == AMP_ACT_TANH, &a, (hipStream_t)hip_stream));
}

int amp_distill_workspace(int dtype, size_t rows, size_t classes, size_t* bytes) {
  const char* what = "distill_workspace";
  CHECK(check_size(what, dtype, rows, classes, "classes"));
  REQUIRE(bytes);
  *bytes = amp_distill_workspace_bytes(dtype, rows, classes);
  return AMP_OK;
}

int amp_distill_loss(int dtype, size_t rows, size_t classes, const void* logits, size_t logits_stride, size_t top, int teacher_dtype,
                     const void* teacher, size_t teacher_stride, const void* index, int index_bytes, size_t index_stride,
                     float temperature, const float* weight, float* loss, void* dlogits, size_t dlogits_stride, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
  const char* what = "distill_loss";
  CHECK(check_size(what, dtype, rows, classes, "classes"));
  if (teacher_dtype < AMP_F32 || teacher_dtype > AMP_F16) return fail(AMP_EINVAL, "%s: unknown teacher_dtype %d", what, teacher_dtype);
  if (index_bytes != 4 && index_bytes != 8) return fail(AMP_EINVAL, "%s: index_bytes %d, 4 and 8 are taken", what, index_bytes);
  if (top < 1 || top > OPS_MAX_TOP) return fail(AMP_EINVAL, "%s: top = %zu, 1 .. %d are taken", what, top, OPS_MAX_TOP);
  // the bounds keep 1 / temperature and temperature^2 in range
  if (!(temperature >= 1e-6f && temperature <= 1e6f)) return fail(AMP_EINVAL, "%s: temperature %g, 1e-6 .. 1e6 are taken", what, temperature);
  if (rows == 0 || (!loss && !dlogits)) return AMP_OK;
  REQUIRE(logits);
  REQUIRE(teacher);
  REQUIRE(index);
  const size_t e = elem(dtype), need = amp_distill_workspace_bytes(dtype, rows, classes);
  const Span s[] = {{"dlogits", dlogits, rows, classes, dlogits_stride, e},
                    {"loss", loss, 1, rows, rows, 4},
                    {"workspace", need ? workspace : nullptr, 1, need, need, 1},
                    {"logits", logits, rows, classes, logits_stride, e},
                    {"teacher", teacher, rows, top, teacher_stride, elem(teacher_dtype)},
                    {"index", index, rows, top, index_stride, (size_t)index_bytes},
                    {"weight", weight, 1, rows, rows, 4}};
  CHECK(check_arrays(what, s, 3));
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  const int pair[][2] = {{0, 3}};
  CHECK(check_overlaps(what, s, 3, pair, 1));
  DistillArgs a = {};
  a.rows = rows, a.classes = classes, a.logits = logits, a.logits_stride = logits_stride, a.top = (int)top;
  a.teacher_dtype = teacher_dtype, a.index_bytes = index_bytes, a.teacher = teacher, a.index = index;
  a.teacher_stride = teacher_stride, a.index_stride = index_stride, a.temperature = temperature, a.weight = weight;
  a.loss = loss, a.dlogits = dlogits, a.dlogits_stride = dlogits_stride, a.workspace = workspace;
  return launched(what, amp_distill_launch(dtype, &a, (hipStream_t)hip_stream));
}

}  // extern "C"
