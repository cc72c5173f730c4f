// Layer norm, forward and backward (include/amp.h has the formulas).
#include "amp_ops.hip.h"

namespace {

constexpr int TPB = 256, NW = TPB / 64;

// One workgroup a row at a time; the row is read again for each of mean, deviations and result.
template <class T>
__global__ __launch_bounds__(TPB) void norm_forward_kernel(NormArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ float part[2][NW][1];
  const long cols = (long)a.cols;
  for (size_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = row_of((const T*)a.x, r, a.x_stride);
    T* y = row_of((T*)a.y, r, a.y_stride);
    float s[1] = {0.f};
    for (long c = threadIdx.x * N; c < cols; c += TPB * N) {
      const Vec<T> v = load_vec(x + c, cols - c);
#pragma unroll
      for (int k = 0; k < N; ++k) s[0] += get(v, k);
    }
    block_sum<NW>(s, part[0]);
    const float mean = s[0] / (float)cols;
    float q[1] = {0.f};
    for (long c = threadIdx.x * N; c < cols; c += TPB * N) {
      const Vec<T> v = load_vec(x + c, cols - c);
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (c + k < cols) q[0] = fmaf(get(v, k) - mean, get(v, k) - mean, q[0]);
    }
    block_sum<NW>(q, part[1]);
    const float rstd = 1.f / sqrtf(q[0] / (float)cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (long c = threadIdx.x * N; c < cols; c += TPB * N) {
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
__global__ __launch_bounds__(TPB) void norm_dx_kernel(NormArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ float part[2][NW][2];
  const long cols = (long)a.cols;
  int turn = 0;
  for (size_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const T* x = row_of((const T*)a.x, r, a.x_stride);
    const T* dy = row_of((const T*)a.dy, r, a.dy_stride);
    T* dx = row_of((T*)a.dx, r, a.dx_stride);
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.f, 0.f};
    for (long c = threadIdx.x * N; c < cols; c += TPB * N) {
      const Vec<T> v = load_vec(x + c, cols - c), g = load_vec(dy + c, cols - c);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float q = get(g, k) * (a.weight && c + k < cols ? a.weight[c + k] : 1.f);
        s[0] += q;
        if (c + k < cols) s[1] = fmaf(q, (get(v, k) - mean) * rstd, s[1]);
      }
    }
    block_sum<NW>(s, part[turn]);
    const float m0 = s[0] / (float)cols, m1 = s[1] / (float)cols;
    for (long c = threadIdx.x * N; c < cols; c += TPB * N) {
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

// Partial sums of the parameters' gradients: block (column group, row part).
template <class T>
__global__ __launch_bounds__(TPB) void norm_dw_kernel(NormArgs a, int parts) {
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

__global__ __launch_bounds__(TPB) void norm_join_kernel(NormArgs a, int parts) {
  const size_t c = (size_t)blockIdx.x * TPB + threadIdx.x;
  if (c >= a.cols) return;
  float w = 0.f, b = 0.f;
  for (int p = 0; p < parts; ++p) {
    w += a.workspace[(size_t)p * 2 * a.cols + c];
    b += a.workspace[((size_t)p * 2 + 1) * a.cols + c];
  }
  if (a.dweight) a.dweight[c] = w;
  if (a.dbias) a.dbias[c] = b;
}

int norm_parts(size_t rows) { return (int)(rows < 64 ? rows : 64); }

}  // namespace

extern "C" size_t amp_norm_workspace_bytes(int, size_t rows, size_t cols) { return (size_t)norm_parts(rows) * 2 * cols * sizeof(float); }

extern "C" hipError_t amp_norm_forward_launch(int dtype, const NormArgs* a, hipStream_t stream) {
  const dim3 grid((unsigned)(a->rows < 65536 ? a->rows : 65536));
  OPS_BY_TYPE(dtype, return launch(norm_forward_kernel<T>, grid, dim3(TPB), 0, stream, *a));
}

extern "C" hipError_t amp_norm_backward_launch(int dtype, const NormArgs* a, hipStream_t stream) {
  const dim3 grid((unsigned)(a->rows < 65536 ? a->rows : 65536));
  const unsigned cb = (unsigned)((a->cols + TPB - 1) / TPB);
  const int parts = norm_parts(a->rows);
  hipError_t e = hipSuccess;
  if (a->dweight || a->dbias) {   // before dx, which may take dy's or x's place
    if (parts) OPS_BY_TYPE(dtype, e = launch(norm_dw_kernel<T>, dim3(cb, parts), dim3(TPB), 0, stream, *a, parts));
    if (e == hipSuccess) e = launch(norm_join_kernel, dim3(cb), dim3(TPB), 0, stream, *a, parts);
  }
  if (e == hipSuccess && a->dx && a->rows) OPS_BY_TYPE(dtype, e = launch(norm_dx_kernel<T>, grid, dim3(TPB), 0, stream, *a));
  return e;
}
