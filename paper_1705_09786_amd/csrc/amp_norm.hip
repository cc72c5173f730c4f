// Layer norm, forward and backward (include/amp.h has the formulas).
//
// Both directions are bound by HBM: a row of up to 32,768 16-bit or 16,384 32-bit elements (16,384 of either backward) is read once and
// stays in the registers of the threads that share it, mean and deviations are formed from there (deviations from the mean itself, not
// as a difference of two sums, which would lose what a mean far from zero leaves), and the backward pass adds the parameters' gradients
// up in registers over all rows of a workgroup. 32,768 x 4,096 bf16: 98 us forward (5.5 TB/s, a large copy's rate), 160 backward (5.0)
// and 4 that join the workgroups' parts; 2,500 x 11,111 fp16, whose rows are not aligned to the groups they are read in: 35 us forward
// (3.2).  Longer rows are read three times in either direction: 4,096 x 40,000 bf16 takes 622 us forward and 845 backward, 5 and 4.4
// times a copy of what they cannot do without.
#include "amp_ops.hip.h"

namespace {

constexpr int TPB = 256;

// Where a thread's groups of a row lie.  TPR threads share a row, thread l has the groups l, l + TPR, ...; the row's last group, where it
// would pass the row's end, is moved back to end with it, and the elements that the group in front of it has as well do not count
// (but are written: the same bits).  Rows shorter than a group are read element by element.
template <class T, int TPR, int NV>
struct Row {
  static constexpr int N = Vec<T>::N;
  int lane, tail, last;   // last: the row's last group is among the threads' group number `last`; tail: elements of it that count
  unsigned mask;          // which elements of group number `last` count in this thread, 0 where it has none
  long cols;
  __device__ explicit Row(size_t cols_) : cols((long)cols_) {
    lane = threadIdx.x % TPR;
    const long groups = (cols + N - 1) / N;
    last = (int)((groups - 1) / TPR);
    const long g = (long)last * TPR + lane, c = g * N;
    mask = g >= groups ? 0 : c + N <= cols ? (1u << N) - 1 : cols >= N ? ((1u << N) - 1) & ~((1u << (c + N - cols)) - 1) : (1u << cols) - 1;
  }
  // the first element of group j (of a thread without one: a group that is there)
  __device__ long at(int j) const {
    const long c = ((long)j * TPR + lane) * N;
    return cols < N ? 0 : c + N <= cols ? c : cols - N;
  }
  __device__ bool counts(int j, int k) const { return j < last || (mask >> k & 1); }
  __device__ Vec<T> load(const T* row, int j) const { return load_vec(row + at(j), cols < N ? cols : N); }
  __device__ void store(T* row, int j, const float (&v)[N]) const {
    if (j < last || mask) store_vec(row + at(j), pack<T>(v), cols < N ? cols : N);
  }
  __device__ void load_param(const float* p, float one, int j, float (&w)[N]) const {
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      Vec<float> v = {(v4u)0u};
      if (p) v = load_vec(p + at(j) + k, cols < N ? cols - k : 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[k + i] = p ? get(v, i) : one;
    }
  }
};

// Sums over the TPR threads of a row, the same bits in each.
template <int TPR, int TPBN, int M>
__device__ __forceinline__ void row_sum(float (&v)[M], float (*part)[M]) {
  if constexpr (TPR <= 64) {
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = group_sum<TPR>(v[m]);
  } else {
    static_assert(TPR == TPBN, "a row to a workgroup");
    block_sum<TPBN / 64>(v, part);
  }
}

template <class T, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_forward_kernel(NormArgs a) {
  constexpr int N = Vec<T>::N, TPBN = TPR > 256 ? TPR : 256, RPW = TPBN / TPR;
  __shared__ float part[2][TPBN / 64][1];
  const Row<T, TPR, NV> R(a.cols);
  constexpr bool KEEP = TPR * NV <= 2048;   // a workgroup has few of the longest rows, and its threads no registers left
  float w[NV][N], b[NV][N];
  if constexpr (KEEP)
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last) {
        R.load_param(a.weight, 1.f, j, w[j]);
        R.load_param(a.bias, 0.f, j, b[j]);
      }
  const float inv = 1.f / (float)a.cols;
  const size_t step = (size_t)gridDim.x * RPW;
  Vec<T> ahead[NV];   // the next row, on its way while this one is worked on
  const auto fetch = [&](size_t r0) {
    const size_t r = r0 + threadIdx.x / TPR;
    const T* x = row_of((const T*)a.x, r < a.rows ? r : a.rows - 1, a.x_stride);
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last) ahead[j] = R.load(x, j);
  };
  fetch((size_t)blockIdx.x * RPW);
  for (size_t r0 = (size_t)blockIdx.x * RPW; r0 < a.rows; r0 += step) {
    const size_t r = r0 + threadIdx.x / TPR;
    const bool in = r < a.rows;
    Vec<T> v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = ahead[j];
    if (r0 + step < a.rows) fetch(r0 + step);
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last)
#pragma unroll
        for (int k = 0; k < N; ++k) s[0] += R.counts(j, k) ? get(v[j], k) : 0.f;
    row_sum<TPR, TPBN>(s, part[0]);
    const float mean = s[0] * inv;
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last)
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float d = R.counts(j, k) ? get(v[j], k) - mean : 0.f;
          q[0] = fmaf(d, d, q[0]);
        }
    row_sum<TPR, TPBN>(q, part[1]);
    const float rstd = 1.f / sqrtf(fmaf(q[0], inv, a.eps));
    if (in) {
      if (R.lane == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
      }
      T* y = row_of((T*)a.y, r, a.y_stride);
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (j <= R.last) {
          float o[N];
          if constexpr (!KEEP) {
            R.load_param(a.weight, 1.f, j, w[j]);
            R.load_param(a.bias, 0.f, j, b[j]);
          }
#pragma unroll
          for (int k = 0; k < N; ++k) o[k] = fmaf((get(v[j], k) - mean) * rstd, w[j][k], b[j][k]);
          R.store(y, j, o);
        }
    }
  }
}

// dx, and the workgroup's part of dweight and dbias into row blockIdx.x of the workspace (2 x cols floats).
template <class T, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_backward_kernel(NormArgs a) {
  constexpr int N = Vec<T>::N, TPBN = TPR > 256 ? TPR : 256, RPW = TPBN / TPR;
  __shared__ float part[2][TPBN / 64][2];
  const Row<T, TPR, NV> R(a.cols);
  float w[NV][N], dw[NV][N], db[NV][N];
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j <= R.last) {
      R.load_param(a.weight, 1.f, j, w[j]);
#pragma unroll
      for (int k = 0; k < N; ++k) dw[j][k] = db[j][k] = 0.f;
    }
  const float inv = 1.f / (float)a.cols;
  const size_t step = (size_t)gridDim.x * RPW;
  constexpr bool AHEAD = TPR * NV <= 2048;   // longer rows leave no registers for a second one
  Vec<T> ahead_x[NV], ahead_dy[NV];          // the next row, on its way while this one is worked on
  float ahead_mean, ahead_rstd;
  const auto fetch = [&](size_t r0) {
    const size_t r = r0 + threadIdx.x / TPR, rr = r < a.rows ? r : a.rows - 1;
    const T *x = row_of((const T*)a.x, rr, a.x_stride), *dy = row_of((const T*)a.dy, rr, a.dy_stride);
    ahead_mean = a.mean[rr], ahead_rstd = a.rstd[rr];
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last) {
        ahead_x[j] = R.load(x, j);
        ahead_dy[j] = R.load(dy, j);
      }
  };
  fetch((size_t)blockIdx.x * RPW);
  int turn = 0;
  for (size_t r0 = (size_t)blockIdx.x * RPW; r0 < a.rows; r0 += step, turn ^= 1) {
    const size_t r = r0 + threadIdx.x / TPR;
    const bool in = r < a.rows;
    Vec<T> v[NV], g[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = ahead_x[j], g[j] = ahead_dy[j];
    const float mean = ahead_mean, rstd = ahead_rstd;
    if (AHEAD && r0 + step < a.rows) fetch(r0 + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last)
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float d = get(g[j], k), n = (get(v[j], k) - mean) * rstd, q = R.counts(j, k) ? d * w[j][k] : 0.f;
          s[0] += q;
          s[1] += R.counts(j, k) ? q * n : 0.f;
          if (in) {
            dw[j][k] = fmaf(d, n, dw[j][k]);
            db[j][k] += d;
          }
        }
    if (a.dx) {
      row_sum<TPR, TPBN>(s, part[turn]);
      const float m0 = s[0] * inv, m1 = s[1] * inv;
      if (in) {
        T* dx = row_of((T*)a.dx, r, a.dx_stride);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (j <= R.last) {
            float o[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
              const float n = (get(v[j], k) - mean) * rstd;
              o[k] = rstd * (fmaf(get(g[j], k), w[j][k], -m0) - n * m1);
            }
            R.store(dx, j, o);
          }
      }
    }
    if (!AHEAD && r0 + step < a.rows) fetch(r0 + step);
  }
  if (!a.dweight && !a.dbias) return;
  // the rows that the workgroup's waves have side by side are joined first, in their order
  float *out_w = a.workspace + (size_t)blockIdx.x * 2 * a.cols, *out_b = out_w + a.cols;
  if (gridDim.x == 1) out_w = a.dweight, out_b = a.dbias;   // the only part is the sum
  if constexpr (RPW == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last)
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (R.counts(j, k)) {
            if (out_w) out_w[R.at(j) + k] = dw[j][k];
            if (out_b) out_b[R.at(j) + k] = db[j][k];
          }
  } else {
    constexpr int SPAN = TPR * N;   // columns of a group number
    __shared__ float both[2][RPW][SPAN];
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= R.last) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
          both[0][threadIdx.x / TPR][R.lane * N + k] = dw[j][k];
          both[1][threadIdx.x / TPR][R.lane * N + k] = db[j][k];
        }
        __syncthreads();
        if (threadIdx.x / TPR == 0)
#pragma unroll
          for (int k = 0; k < N; ++k)
            if (R.counts(j, k)) {
              float sw = 0.f, sb = 0.f;
#pragma unroll
              for (int i = 0; i < RPW; ++i) {
                sw += both[0][i][R.lane * N + k];
                sb += both[1][i][R.lane * N + k];
              }
              if (out_w) out_w[R.at(j) + k] = sw;
              if (out_b) out_b[R.at(j) + k] = sb;
            }
      }
  }
}

// Longer rows than the registers hold: one workgroup a row at a time, read again for each of mean, deviations and result (backward:
// for the parameters' gradients, the row's two sums, and dx).
constexpr int LONG = 1024;
template <class T>
__global__ __launch_bounds__(LONG) void norm_forward_long_kernel(NormArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ float part[2][LONG / 64][1];
  const long cols = (long)a.cols;
  for (size_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = row_of((const T*)a.x, r, a.x_stride);
    T* y = row_of((T*)a.y, r, a.y_stride);
    float s[1] = {0.f};
    for (long c = threadIdx.x * N; c < cols; c += LONG * N) {
      const Vec<T> v = load_vec(x + c, cols - c);
#pragma unroll
      for (int k = 0; k < N; ++k) s[0] += get(v, k);
    }
    block_sum<LONG / 64>(s, part[0]);
    const float mean = s[0] / (float)cols;
    float q[1] = {0.f};
    for (long c = threadIdx.x * N; c < cols; c += LONG * N) {
      const Vec<T> v = load_vec(x + c, cols - c);
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (c + k < cols) q[0] = fmaf(get(v, k) - mean, get(v, k) - mean, q[0]);
    }
    block_sum<LONG / 64>(q, part[1]);
    const float rstd = 1.f / sqrtf(q[0] / (float)cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (long c = threadIdx.x * N; c < cols; c += LONG * N) {
      const Vec<T> v = load_vec(x + c, cols - c);
      float o[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const bool in = c + k < cols;
        o[k] = fmaf((get(v, k) - mean) * rstd, a.weight && in ? a.weight[c + k] : 1.f, a.bias && in ? a.bias[c + k] : 0.f);
      }
      store_vec(y + c, pack<T>(o), cols - c);
    }
  }
}

template <class T>
__global__ __launch_bounds__(LONG) void norm_dx_long_kernel(NormArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ float part[2][LONG / 64][2];
  const long cols = (long)a.cols;
  int turn = 0;
  for (size_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const T* x = row_of((const T*)a.x, r, a.x_stride);
    const T* dy = row_of((const T*)a.dy, r, a.dy_stride);
    T* dx = row_of((T*)a.dx, r, a.dx_stride);
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.f, 0.f};
    for (long c = threadIdx.x * N; c < cols; c += LONG * N) {
      const Vec<T> v = load_vec(x + c, cols - c), g = load_vec(dy + c, cols - c);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float q = get(g, k) * (a.weight && c + k < cols ? a.weight[c + k] : 1.f);
        s[0] += q;
        if (c + k < cols) s[1] = fmaf(q, (get(v, k) - mean) * rstd, s[1]);
      }
    }
    block_sum<LONG / 64>(s, part[turn]);
    const float m0 = s[0] / (float)cols, m1 = s[1] / (float)cols;
    for (long c = threadIdx.x * N; c < cols; c += LONG * N) {
      const Vec<T> v = load_vec(x + c, cols - c), g = load_vec(dy + c, cols - c);
      float o[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float q = get(g, k) * (a.weight && c + k < cols ? a.weight[c + k] : 1.f);
        o[k] = rstd * (q - m0 - (get(v, k) - mean) * rstd * m1);
      }
      store_vec(dx + c, pack<T>(o), cols - c);
    }
  }
}

// Partial sums of the parameters' gradients: block (columns, row part).
template <class T>
__global__ __launch_bounds__(TPB) void norm_dw_long_kernel(NormArgs a, int parts) {
  const size_t c = (size_t)blockIdx.x * TPB + threadIdx.x;
  if (c >= a.cols) return;
  float w = 0.f, b = 0.f;
  for (size_t r = blockIdx.y; r < a.rows; r += parts) {
    const float g = widen(row_of((const T*)a.dy, r, a.dy_stride)[c]);
    w = fmaf(g, (widen(row_of((const T*)a.x, r, a.x_stride)[c]) - a.mean[r]) * a.rstd[r], w);
    b += g;
  }
  a.workspace[(size_t)blockIdx.y * 2 * a.cols + c] = w;
  a.workspace[((size_t)blockIdx.y * 2 + 1) * a.cols + c] = b;
}

// The parts' sums, in their order within each of JOIN shares of them, and the shares': 32 columns to a workgroup.  A launch takes fewer
// than 2^32 threads in a line (and starts fewer without an error where there are more), so the workgroups have several lines.
constexpr int JOIN = 32;
constexpr size_t JOIN_LINE = (size_t)1 << 20;
__global__ __launch_bounds__(32 * JOIN) void norm_join_kernel(NormArgs a, int parts) {
  __shared__ float sum[JOIN][33];
  const int lane = threadIdx.x % 32, share = threadIdx.x / 32;
  const size_t c = ((size_t)blockIdx.y * JOIN_LINE + blockIdx.x) * 32 + lane, cols2 = 2 * a.cols;
  float s = 0.f;
  if (c < cols2)
    for (int p = share; p < parts; p += 8 * JOIN) {
      float v[8];   // on their way together
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = p + i * JOIN < parts ? a.workspace[(size_t)(p + i * JOIN) * cols2 + c] : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
  sum[share][lane] = s;
  __syncthreads();
  if (share == 0 && c < cols2) {
    s = 0.f;
    for (int i = 0; i < JOIN; ++i) s += sum[i][lane];
    float* out = c < a.cols ? a.dweight : a.dbias;
    if (out) out[c < a.cols ? c : c - a.cols] = s;
  }
}

// Which kernel takes a row: the threads that share it and the 16-byte groups of each.  A wave to a row of up to 128 groups (256
// forward) has no barriers; longer rows, and rows so few that a call is a latency (512 and fewer), have more threads.  The backward pass
// keeps three values a column beside the row, so its threads have fewer groups: 2,500 x 11,111 fp16 takes 70 us on 1,024 threads of
// two, 61 on 512 of four (forward, of inputs that the memory-side cache holds, 33 and 38).  Its workgroups, of which each leaves a part of
// the parameters' gradients to be read again, have at least eight rows: 512 x 4,096 bf16 takes 27 us with a row to each, 2,048 x 4,096 43 us
// and 27 with eight.
struct Shape {
  int tpr, nv, parts;   // tpr = 0: longer than the registers hold; parts: workgroups of the backward pass
};
Shape shape_of(int dtype, size_t rows, size_t cols, bool backward) {
  const size_t groups = (cols * (dtype == 0 ? 4 : 2) + 15) / 16;
  Shape s = {0, 0, 0};
  if (groups <= 16) s = {16, 1, 0};
  else if (groups <= 64) s = {64, 1, 0};
  else if (groups <= 256 && (backward ? groups > 128 || rows <= 512 : rows <= 512)) s = {256, 1, 0};
  else if (groups <= 128) s = {64, 2, 0};
  else if (groups <= 256) s = {64, 4, 0};
  else if (groups <= 512) s = {256, 2, 0};
  else if (groups <= 1024) s = backward ? Shape{1024, 1, 0} : Shape{256, 4, 0};
  else if (groups <= 2048) s = backward ? Shape{512, 4, 0} : Shape{1024, 2, 0};
  else if (groups <= 4096 && (!backward || dtype == 0)) s = {1024, 4, 0};
  const size_t rpw = s.tpr && s.tpr < 256 ? 256 / s.tpr : 1, most = s.tpr == 0 ? 64 : s.tpr > 256 ? 256 : 512;
  const size_t need = (rows + rpw * 8 - 1) / (rpw * 8);
  s.parts = (int)(need < most ? need : most);
  return s;
}

#define NORM_SHAPES(K)                                   \
  switch (s.tpr * 8 + s.nv) {                            \
    case 16 * 8 + 1: return K(16, 1);                    \
    case 64 * 8 + 1: return K(64, 1);                    \
    case 64 * 8 + 2: return K(64, 2);                    \
    case 256 * 8 + 1: return K(256, 1);                  \
    case 256 * 8 + 2: return K(256, 2);

template <class T>
hipError_t forward(const Shape& s, const NormArgs* a, hipStream_t stream) {
  const size_t rpw = s.tpr && s.tpr < 256 ? 256 / s.tpr : 1, need = (a->rows + rpw - 1) / rpw;
#define NORM_F(TPR, NV) \
  launch(norm_forward_kernel<T, TPR, NV>, dim3((unsigned)(need < 768 ? need : 768)), dim3(TPR > 256 ? TPR : 256), 0, stream, *a)
  NORM_SHAPES(NORM_F)
    case 64 * 8 + 4: return NORM_F(64, 4);
    case 256 * 8 + 4: return NORM_F(256, 4);
    case 1024 * 8 + 2: return NORM_F(1024, 2);
    case 1024 * 8 + 4: return NORM_F(1024, 4);
    default: return launch(norm_forward_long_kernel<T>, dim3((unsigned)(a->rows < 4096 ? a->rows : 4096)), dim3(LONG), 0, stream, *a);
  }
}

template <class T>
hipError_t backward(const Shape& s, const NormArgs* a, hipStream_t stream) {
#define NORM_B(TPR, NV) launch(norm_backward_kernel<T, TPR, NV>, dim3((unsigned)s.parts), dim3(TPR > 256 ? TPR : 256), 0, stream, *a)
  NORM_SHAPES(NORM_B)
    case 512 * 8 + 4: return NORM_B(512, 4);
    case 1024 * 8 + 1: return NORM_B(1024, 1);
    default: break;
  }
  if constexpr (sizeof(T) == 4)
    if (s.tpr == 1024 && s.nv == 4) return NORM_B(1024, 4);
  if (a->dweight || a->dbias) {   // before dx, which may take dy's or x's place
    const hipError_t e = launch(norm_dw_long_kernel<T>, dim3((unsigned)((a->cols + TPB - 1) / TPB), (unsigned)s.parts), dim3(TPB), 0, stream, *a, s.parts);
    if (e != hipSuccess || !a->dx) return e;
  }
  return launch(norm_dx_long_kernel<T>, dim3((unsigned)(a->rows < 4096 ? a->rows : 4096)), dim3(LONG), 0, stream, *a);
}

}  // namespace

extern "C" size_t amp_norm_workspace_bytes(int dtype, size_t rows, size_t cols) {
  const Shape s = shape_of(dtype, rows, cols, true);
  return s.tpr && s.parts == 1 ? 0 : ((size_t)s.parts * 2 * cols * sizeof(float) + 15) / 16 * 16;
}

extern "C" hipError_t amp_norm_forward_launch(int dtype, const NormArgs* a, hipStream_t stream) {
  const Shape s = shape_of(dtype, a->rows, a->cols, false);
  OPS_BY_TYPE(dtype, return forward<T>(s, a, stream));
}

extern "C" hipError_t amp_norm_backward_launch(int dtype, const NormArgs* a, hipStream_t stream) {
  const Shape s = shape_of(dtype, a->rows, a->cols, true);
  hipError_t e = hipSuccess;
  if (a->rows) OPS_BY_TYPE(dtype, e = backward<T>(s, a, stream));
  if (e == hipSuccess && (a->dweight || a->dbias) && !(s.tpr && s.parts == 1)) {
    const size_t groups = (2 * a->cols + 31) / 32, line = groups < JOIN_LINE ? groups : JOIN_LINE;
    e = launch(norm_join_kernel, dim3((unsigned)line, (unsigned)((groups + line - 1) / line)), dim3(32 * JOIN), 0, stream, *a, a->rows ? s.parts : 0);
  }
  return e;
}
