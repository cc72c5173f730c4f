// C entry points of the operators on whole arrays (include/amp.h): argument checks and launches.  Nothing here allocates (but a list of host
// memory, while clipping's results are checked), waits or throws.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>

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

// The recurrences' kernels reach a tile's rows by 32-bit offsets.
int check_scan_stride(const char* what, const char* name, size_t stride) {
  return stride < (size_t)1 << 22 ? AMP_OK : fail(AMP_EINVAL, "%s: %s has a row stride of 2^22 or more", what, name);
}

int check_sequences(const char* what, const amp_sequences* q) {
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

int check_scan(const char* what, int dtype, int activation, size_t rows, size_t hidden, const amp_sequences* q) {
  CHECK(check_scan_size(what, dtype, rows, hidden));
  if (activation != AMP_ACT_NONE && activation != AMP_ACT_TANH)
    return fail(AMP_EINVAL, "%s: activation %d, AMP_ACT_NONE and AMP_ACT_TANH are taken", what, activation);
  return check_sequences(what, q);
}

#define REQUIRE(p)                                                              \
  do {                                                                          \
    if (!(p)) return fail(AMP_EINVAL, "%s: %s is NULL", what, #p);              \
  } while (0)

int check_delta_shape(const char* what, const amp_delta_shape* s, size_t n) {
  if (!s) return fail(AMP_EINVAL, "%s: shape is NULL", what);
  if (s->dtype < AMP_F32 || s->dtype > AMP_F16) return fail(AMP_EINVAL, "%s: unknown dtype %d", what, s->dtype);
  if (s->rows >= MAX_ROWS / 2) return fail(AMP_EINVAL, "%s: %zu rows, fewer than 2^30 are taken", what, s->rows);
  if (s->heads < 1 || s->heads >= (size_t)1 << 16) return fail(AMP_EINVAL, "%s: heads = %zu, 1 .. 65535 are taken", what, s->heads);
  if (s->key_heads < 1 || s->key_heads > s->heads || s->heads % s->key_heads)
    return fail(AMP_EINVAL, "%s: key_heads = %zu does not divide heads = %zu", what, s->key_heads, s->heads);
  if (s->dk < 1 || s->dk > DELTA_MAX_KEY) return fail(AMP_EINVAL, "%s: dk = %zu, 1 .. %d are taken", what, s->dk, DELTA_MAX_KEY);
  if (s->dv < 1 || s->dv > 1024) return fail(AMP_EINVAL, "%s: dv = %zu, 1 .. 1024 are taken", what, s->dv);
  if (n >= MAX_ROWS) return fail(AMP_EINVAL, "%s: %zu sequences, fewer than 2^31 are taken", what, n);
  if (s->heads * s->dv >= (size_t)1 << 22 || s->key_heads * s->dk >= (size_t)1 << 22)
    return fail(AMP_EINVAL, "%s: rows of heads x dv or key_heads x dk = 2^22 elements or more", what);
  // a launch has fewer than 2^32 threads, a workgroup to a block or a sequence, and a head
  if ((s->rows / DELTA_BLOCK + n) * s->heads > (size_t)1 << 22)
    return fail(AMP_EINVAL, "%s: %zu rows in %zu sequences of %zu heads, up to 2^22 of (rows / %d + sequences) heads are taken", what, s->rows, n,
                s->heads, DELTA_BLOCK);
  return AMP_OK;
}

// What the calls of the delta rule have in common, in front of their outputs.
struct DeltaIn {
  const void* p;
  size_t stride;
};
void delta_in(DeltaArgs& a, const amp_delta_shape* s, const DeltaIn& q, const DeltaIn& k, const DeltaIn& v, const DeltaIn& decay, const DeltaIn& beta,
              float scale, const amp_sequences* seq) {
  a.rows = s->rows, a.heads = (int)s->heads, a.key_heads = (int)s->key_heads, a.dk = (int)s->dk, a.dv = (int)s->dv;
  a.q = q.p, a.q_stride = q.stride, a.k = k.p, a.k_stride = k.stride, a.v = v.p, a.v_stride = v.stride;
  a.decay = (const float*)decay.p, a.decay_stride = decay.stride, a.beta = (const float*)beta.p, a.beta_stride = beta.stride, a.scale = scale;
  a.n_seq = seq->n, a.begin = seq->begin, a.end = seq->end, a.index_bytes = seq->index_bytes, a.zero_others = seq->zero_others;
}

size_t delta_carry_floats(const amp_delta_shape* s, size_t n) {
  return amp_delta_blocks(s->rows, n) * s->heads * (DELTA_BLOCK + s->dk) * ((s->dv + 15) / 16 * 16);
}

constexpr size_t MAX_TENSORS = (size_t)1 << 20, MAX_ELEMENTS = (size_t)1 << 40;

static_assert(sizeof(ClipTensor) == sizeof(amp_tensor) && offsetof(ClipTensor, dtype) == offsetof(amp_tensor, dtype), "one layout");

int check_tensors(const char* what, size_t n, const amp_tensor* t) {
  if (n > MAX_TENSORS) return fail(AMP_EINVAL, "%s: %zu tensors, up to 2^20 are taken", what, n);
  if (n && !t) return fail(AMP_EINVAL, "%s: tensors is NULL", what);
  size_t total = 0;
  for (size_t i = 0; i < n; ++i) {
    if (t[i].dtype < AMP_F32 || t[i].dtype > AMP_F16) return fail(AMP_EINVAL, "%s: tensor %zu: unknown dtype %d", what, i, t[i].dtype);
    if (t[i].n > MAX_ELEMENTS || (total += t[i].n) > MAX_ELEMENTS) return fail(AMP_EINVAL, "%s: more than 2^40 elements", what);
    if (!t[i].n) continue;
    if (!t[i].p) return fail(AMP_EINVAL, "%s: tensor %zu is NULL", what, i);
    if (((uintptr_t)t[i].p | (uintptr_t)t[i].out) % elem(t[i].dtype))
      return fail(AMP_EINVAL, "%s: tensor %zu is not aligned to its elements", what, i);
  }
  return AMP_OK;
}

// Memory that a tensor is read from, or its result written to.
struct Range {
  uintptr_t first, last;
  size_t tensor;   // -1: the norm or the workspace
  bool written;
};

// No result overlaps anything but its own tensor, and that only as a whole.
int check_results(const char* what, size_t n, const amp_tensor* t, const float* norm, const void* ws, size_t need) {
  // as most lists are: the results one behind the other in a buffer of their own, none of the tensors in it
  uintptr_t from = UINTPTR_MAX, to = 0;
  bool plain = true;
  const auto outside = [&](const void* p, size_t bytes) { return !p || !bytes || (uintptr_t)p >= to || (uintptr_t)p + bytes <= from; };
  for (size_t i = 0; i < n && plain; ++i)
    if (t[i].n && t[i].out) {
      plain = t[i].out != t[i].p && (uintptr_t)t[i].out >= to;
      from = std::min(from, (uintptr_t)t[i].out), to = (uintptr_t)t[i].out + t[i].n * elem(t[i].dtype);
    }
  for (size_t i = 0; i < n && plain; ++i) {
    const size_t bytes = t[i].n * elem(t[i].dtype);
    plain = outside(t[i].p, bytes) && ((uintptr_t)norm >= (uintptr_t)t[i].p + bytes || (uintptr_t)norm + sizeof(float) <= (uintptr_t)t[i].p) &&
            ((uintptr_t)ws >= (uintptr_t)t[i].p + bytes || (uintptr_t)ws + need <= (uintptr_t)t[i].p);
  }
  if (plain && outside(norm, sizeof(float)) && outside(ws, need) &&
      ((uintptr_t)norm >= (uintptr_t)ws + need || (uintptr_t)norm + sizeof(float) <= (uintptr_t)ws))
    return AMP_OK;
  Range* r = (Range*)malloc((2 * n + 2) * sizeof(Range));
  if (!r) return fail(AMP_ENOMEM, "%s: no host memory for %zu ranges", what, 2 * n + 2);
  size_t m = 0;
  for (size_t i = 0; i < n; ++i) {
    if (!t[i].n) continue;
    const size_t bytes = t[i].n * elem(t[i].dtype);
    r[m++] = {(uintptr_t)t[i].p, (uintptr_t)t[i].p + bytes, i, t[i].p == t[i].out};
    if (t[i].out && t[i].out != t[i].p) r[m++] = {(uintptr_t)t[i].out, (uintptr_t)t[i].out + bytes, i, true};
  }
  if (norm) r[m++] = {(uintptr_t)norm, (uintptr_t)norm + sizeof(float), (size_t)-1, true};
  if (need) r[m++] = {(uintptr_t)ws, (uintptr_t)ws + need, (size_t)-1, true};
  std::sort(r, r + m, [](const Range& a, const Range& b) { return a.first < b.first; });
  // in the order of their beginnings, a range meets one in front of it where that, or one further in front, ends behind its beginning
  uintptr_t any = 0, written = 0;
  size_t bad = m;
  for (size_t i = 0; i < m && bad == m; ++i) {
    if (r[i].first < written || (r[i].written && r[i].first < any)) bad = i;
    any = std::max(any, r[i].last);
    if (r[i].written) written = std::max(written, r[i].last);
  }
  const size_t tensor = bad < m ? r[bad].tensor : 0;
  free(r);
  if (bad == m) return AMP_OK;
  if (tensor == (size_t)-1) return fail(AMP_EINVAL, "%s: norm or workspace overlaps a tensor or a result", what);
  return fail(AMP_EINVAL, "%s: tensor %zu overlaps a result, or its result another tensor", what, tensor);
}

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

int amp_gated_delta_carry(const amp_delta_shape* s, size_t n, size_t* floats) {
  const char* what = "gated_delta_carry";
  CHECK(check_delta_shape(what, s, n));
  REQUIRE(floats);
  *floats = delta_carry_floats(s, n);
  return AMP_OK;
}

int amp_gated_delta_workspace(const amp_delta_shape* s, size_t n, int backward, size_t* bytes) {
  const char* what = "gated_delta_workspace";
  CHECK(check_delta_shape(what, s, n));
  REQUIRE(bytes);
  *bytes = amp_delta_workspace_bytes(s->rows, n, s->heads, s->key_heads, s->dk, s->dv, backward);
  return AMP_OK;
}

int amp_gated_delta_forward(const amp_delta_shape* shape, const void* q, size_t q_stride, const void* k, size_t k_stride, const void* v,
                            size_t v_stride, const float* decay, size_t decay_stride, const float* beta, size_t beta_stride, float scale,
                            const amp_sequences* seq, const float* h0, void* o, size_t o_stride, float* last, float* carry, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  const char* what = "gated_delta_forward";
  CHECK(check_sequences(what, seq));
  CHECK(check_delta_shape(what, shape, seq->n));
  const size_t rows = shape->rows, heads = shape->heads, n = seq->n, ib = seq->index_bytes;
  if ((n == 0 && !seq->zero_others) || (!o && !last && !carry)) return AMP_OK;
  if (rows) {
    REQUIRE(q);
    REQUIRE(k);
    REQUIRE(v);
    REQUIRE(decay);
    REQUIRE(beta);
  }
  const size_t e = elem(shape->dtype), keys = shape->key_heads * shape->dk, values = heads * shape->dv, state = heads * shape->dk * shape->dv;
  const size_t need = amp_delta_workspace_bytes(rows, n, heads, shape->key_heads, shape->dk, shape->dv, 0), nc = delta_carry_floats(shape, n);
  const Span s[] = {{"o", o, rows, values, o_stride, e},          {"last", last, n, state, state, 4},
                    {"carry", carry, 1, nc, nc, 4},               {"workspace", need ? workspace : nullptr, 1, need, need, 1},
                    {"q", q, rows, keys, q_stride, e},            {"k", k, rows, keys, k_stride, e},
                    {"v", v, rows, values, v_stride, e},          {"decay", decay, rows, heads, decay_stride, 4},
                    {"beta", beta, rows, heads, beta_stride, 4},  {"h0", h0, n, state, state, 4},
                    {"begin", seq->begin, 1, n, n, seq->begin ? ib : 1}, {"end", seq->end, 1, n, n, seq->end ? ib : 1}};
  CHECK(check_arrays(what, s, 4));
  if (rows > 1) CHECK(check_scan_stride(what, "q", q_stride));
  if (rows > 1) CHECK(check_scan_stride(what, "k", k_stride));
  if (rows > 1) CHECK(check_scan_stride(what, "v", v_stride));
  if (rows > 1) CHECK(check_scan_stride(what, "o", o_stride));
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  CHECK(check_overlaps(what, s, 4, nullptr, 0));
  DeltaArgs a = {};
  delta_in(a, shape, {q, q_stride}, {k, k_stride}, {v, v_stride}, {decay, decay_stride}, {beta, beta_stride}, scale, seq);
  a.h0 = h0, a.o = o, a.o_stride = o_stride, a.last = last, a.carry = carry, a.workspace = workspace;
  a.zero[0] = {o, o_stride * e, values * e / 2};
  return launched(what, amp_delta_forward_launch(shape->dtype, &a, (hipStream_t)hip_stream));
}

int amp_gated_delta_backward(const amp_delta_shape* shape, const void* dout, size_t dout_stride, const float* dlast, const void* q,
                             size_t q_stride, const void* k, size_t k_stride, const void* v, size_t v_stride, const float* decay,
                             size_t decay_stride, const float* beta, size_t beta_stride, float scale, const amp_sequences* seq,
                             const float* carry, void* dq, size_t dq_stride, void* dk, size_t dk_stride, void* dv, size_t dv_stride,
                             float* ddecay, size_t ddecay_stride, float* dbeta, size_t dbeta_stride, float* dh0, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  const char* what = "gated_delta_backward";
  CHECK(check_sequences(what, seq));
  CHECK(check_delta_shape(what, shape, seq->n));
  const size_t rows = shape->rows, heads = shape->heads, n = seq->n, ib = seq->index_bytes;
  if (n == 0 && !seq->zero_others) return AMP_OK;
  if (rows) {
    REQUIRE(dout);
    REQUIRE(q);
    REQUIRE(k);
    REQUIRE(v);
    REQUIRE(decay);
    REQUIRE(beta);
    if (n) REQUIRE(carry);
    REQUIRE(dq);
    REQUIRE(dk);
    REQUIRE(dv);
    REQUIRE(ddecay);
    REQUIRE(dbeta);
  }
  const size_t e = elem(shape->dtype), keys = shape->key_heads * shape->dk, values = heads * shape->dv, state = heads * shape->dk * shape->dv;
  const size_t need = amp_delta_workspace_bytes(rows, n, heads, shape->key_heads, shape->dk, shape->dv, 1), nc = delta_carry_floats(shape, n);
  const Span s[] = {{"dq", dq, rows, keys, dq_stride, e},               {"dk", dk, rows, keys, dk_stride, e},
                    {"dv", dv, rows, values, dv_stride, e},             {"ddecay", ddecay, rows, heads, ddecay_stride, 4},
                    {"dbeta", dbeta, rows, heads, dbeta_stride, 4},     {"dh0", dh0, n, state, state, 4},
                    {"workspace", need ? workspace : nullptr, 1, need, need, 1},
                    {"dout", dout, rows, values, dout_stride, e},       {"q", q, rows, keys, q_stride, e},
                    {"k", k, rows, keys, k_stride, e},                  {"v", v, rows, values, v_stride, e},
                    {"decay", decay, rows, heads, decay_stride, 4},     {"beta", beta, rows, heads, beta_stride, 4},
                    {"carry", carry, 1, nc, nc, 4},                     {"dlast", dlast, n, state, state, 4},
                    {"begin", seq->begin, 1, n, n, seq->begin ? ib : 1}, {"end", seq->end, 1, n, n, seq->end ? ib : 1}};
  CHECK(check_arrays(what, s, 7));
  if (rows > 1) CHECK(check_scan_stride(what, "dout", dout_stride));
  if (rows > 1) CHECK(check_scan_stride(what, "q", q_stride));
  if (rows > 1) CHECK(check_scan_stride(what, "k", k_stride));
  if (rows > 1) CHECK(check_scan_stride(what, "v", v_stride));
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  CHECK(check_overlaps(what, s, 7, nullptr, 0));
  DeltaArgs a = {};
  delta_in(a, shape, {q, q_stride}, {k, k_stride}, {v, v_stride}, {decay, decay_stride}, {beta, beta_stride}, scale, seq);
  a.dout = dout, a.dout_stride = dout_stride, a.dlast = dlast, a.carry_in = carry, a.workspace = workspace;
  a.dq = dq, a.dq_stride = dq_stride, a.dkey = dk, a.dk_stride = dk_stride, a.dvalue = dv, a.dv_stride = dv_stride;
  a.ddecay = ddecay, a.ddecay_stride = ddecay_stride, a.dbeta = dbeta, a.dbeta_stride = dbeta_stride, a.dh0 = dh0;
  a.zero[0] = {dq, dq_stride * e, keys * e / 2}, a.zero[1] = {dk, dk_stride * e, keys * e / 2}, a.zero[2] = {dv, dv_stride * e, values * e / 2};
  a.zero[3] = {ddecay, ddecay_stride * 4, heads * 2}, a.zero[4] = {dbeta, dbeta_stride * 4, heads * 2};
  return launched(what, amp_delta_backward_launch(shape->dtype, &a, (hipStream_t)hip_stream));
}

int amp_gated_delta_step(const amp_delta_shape* shape, const void* q, size_t q_stride, const void* k, size_t k_stride, const void* v,
                         size_t v_stride, const float* decay, size_t decay_stride, const float* beta, size_t beta_stride, float scale,
                         float* state, size_t state_stride, void* o, size_t o_stride, void* hip_stream) {
  const char* what = "gated_delta_step";
  CHECK(check_delta_shape(what, shape, 0));
  const size_t rows = shape->rows, heads = shape->heads, e = elem(shape->dtype);
  if (rows == 0) return AMP_OK;
  if (rows * heads > (size_t)1 << 22) return fail(AMP_EINVAL, "%s: %zu rows of %zu heads, up to 2^22 are taken", what, rows, heads);
  REQUIRE(q);
  REQUIRE(k);
  REQUIRE(v);
  REQUIRE(decay);
  REQUIRE(beta);
  REQUIRE(state);
  const size_t keys = shape->key_heads * shape->dk, values = heads * shape->dv;
  const Span s[] = {{"state", state, rows, heads * shape->dk * shape->dv, state_stride, 4}, {"o", o, rows, values, o_stride, e},
                    {"q", q, rows, keys, q_stride, e},            {"k", k, rows, keys, k_stride, e},
                    {"v", v, rows, values, v_stride, e},          {"decay", decay, rows, heads, decay_stride, 4},
                    {"beta", beta, rows, heads, beta_stride, 4}};
  CHECK(check_arrays(what, s, 2));
  CHECK(check_overlaps(what, s, 2, nullptr, 0));
  DeltaStepArgs a = {};
  a.rows = rows, a.heads = (int)heads, a.key_heads = (int)shape->key_heads, a.dk = (int)shape->dk, a.dv = (int)shape->dv;
  a.q = q, a.q_stride = q_stride, a.k = k, a.k_stride = k_stride, a.v = v, a.v_stride = v_stride, a.decay = decay, a.decay_stride = decay_stride;
  a.beta = beta, a.beta_stride = beta_stride, a.scale = scale, a.state = state, a.state_stride = state_stride, a.o = o, a.o_stride = o_stride;
  return launched(what, amp_delta_step_launch(shape->dtype, &a, (hipStream_t)hip_stream));
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

int amp_policy_loss(int dtype, size_t rows, size_t classes, const void* logits, size_t logits_stride, const void* index, int index_bytes,
                    double temperature, const float* advantage, const float* old, const float* reference, double kl, double clip_low,
                    double clip_high, const float* weight, float* loss, float* logprob, void* dlogits, size_t dlogits_stride,
                    void* hip_stream) {
  const char* what = "policy_loss";
  CHECK(check_size(what, dtype, rows, classes, "classes"));
  if (index_bytes != 4 && index_bytes != 8) return fail(AMP_EINVAL, "%s: index_bytes %d, 4 and 8 are taken", what, index_bytes);
  if (!(temperature >= 1e-6 && temperature <= 1e6)) return fail(AMP_EINVAL, "%s: temperature %g, 1e-6 .. 1e6 are taken", what, temperature);
  if (!(clip_low >= 0.0 && clip_low <= 1.0)) return fail(AMP_EINVAL, "%s: clip_low %g, 0 .. 1 are taken", what, clip_low);
  if (!(clip_high >= 0.0)) return fail(AMP_EINVAL, "%s: clip_high %g, 0 and more are taken", what, clip_high);
  if (!(fabs(kl) < INFINITY)) return fail(AMP_EINVAL, "%s: kl %g is not finite", what, kl);
  if (rows == 0 || (!loss && !logprob && !dlogits)) return AMP_OK;
  REQUIRE(logits);
  REQUIRE(index);
  if (loss || dlogits) REQUIRE(advantage);
  const size_t e = elem(dtype);
  const Span s[] = {{"dlogits", dlogits, rows, classes, dlogits_stride, e}, {"loss", loss, 1, rows, rows, 4},
                    {"logprob", logprob, 1, rows, rows, 4},                 {"logits", logits, rows, classes, logits_stride, e},
                    {"index", index, 1, rows, rows, (size_t)index_bytes},   {"advantage", advantage, 1, rows, rows, 4},
                    {"old", old, 1, rows, rows, 4},                         {"reference", reference, 1, rows, rows, 4},
                    {"weight", weight, 1, rows, rows, 4}};
  CHECK(check_arrays(what, s, 3));
  const int pair[][2] = {{0, 3}};
  CHECK(check_overlaps(what, s, 3, pair, 1));
  PolicyArgs a = {};
  a.rows = rows, a.classes = classes, a.logits = logits, a.logits_stride = logits_stride, a.index = index, a.index_bytes = index_bytes;
  a.inverse = 1.0 / temperature, a.scale = 1.4426950408889634074 / temperature;
  a.kl = kl, a.low = 1.0 - clip_low, a.high = 1.0 + clip_high, a.log_low = log1p(-clip_low), a.log_high = log1p(clip_high);
  a.advantage = advantage, a.old = old, a.reference = reference, a.weight = weight;
  a.loss = loss, a.logprob = logprob, a.dlogits = dlogits, a.dlogits_stride = dlogits_stride;
  return launched(what, amp_policy_launch(dtype, &a, (hipStream_t)hip_stream));
}

int amp_clip_workspace(size_t n, const amp_tensor* tensors, size_t* bytes) {
  const char* what = "clip_workspace";
  CHECK(check_tensors(what, n, tensors));
  REQUIRE(bytes);
  *bytes = amp_clip_workspace_bytes(n, (const ClipTensor*)tensors);
  return AMP_OK;
}

int amp_clip_gradients(size_t n, const amp_tensor* tensors, double max_norm, float* norm, void* workspace, size_t workspace_bytes,
                       void* hip_stream) {
  const char* what = "clip_gradients";
  CHECK(check_tensors(what, n, tensors));
  if (!(max_norm >= 0.0)) return fail(AMP_EINVAL, "%s: max_norm is negative or not a number", what);
  if ((uintptr_t)norm % sizeof(float)) return fail(AMP_EINVAL, "%s: norm is not aligned to its 4-byte elements", what);
  const size_t need = amp_clip_workspace_bytes(n, (const ClipTensor*)tensors);
  CHECK(check_workspace(what, workspace, workspace_bytes, need));
  CHECK(check_results(what, n, tensors, norm, workspace, need));
  return launched(what, amp_clip_launch(n, (const ClipTensor*)tensors, max_norm, norm, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
