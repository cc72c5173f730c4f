// The norm over many tensors and their clipping (include/amp.h has the formulas).
//
// Bound by HBM: every tensor is read once for the squares and, where there is a result, once more for that. A launch's workgroups take pieces of the
// tensors that its arguments list, each piece's sum of squares has a place of its own in the workspace, in 64 bits (a square of a
// float may be beyond floats, and a sum of 2^30 of them loses half its digits), and one workgroup adds the places up in their order.  The
// second reading goes through the tensors from the last to the first, so that it begins with what the memory-side cache has last seen.
// 97 tensors of 314 million floats together: the norm in 217 us (5.8 TB/s). 600 of 302 million bf16: 400 us a call with results elsewhere, calls back
// to back (147 for the norm and 226 for the results where a profiler lets each of the ten launches wait for the one in front); in place 236
// where the norm is not beyond the limit, as long as the host takes for them.
#include <float.h>

#include "amp_ops.hip.h"

namespace {

constexpr int TPB = 256;

__device__ __forceinline__ int find(const ClipList& l, unsigned piece) {
  int lo = 0, hi = l.n;   // first[lo] <= piece < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (l.first[mid] <= piece) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <class T>
__device__ __forceinline__ double squares(const T* p, size_t n) {
  constexpr int N = Vec<T>::N, DEEP = 4;
  double sum[2] = {0.0, 0.0};
  size_t i = threadIdx.x * N;
  for (; i + (DEEP - 1) * TPB * N + N <= n; i += DEEP * TPB * N) {
    Vec<T> v[DEEP];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) v[j] = load_vec(p + i + (size_t)j * TPB * N, N);
#pragma unroll
    for (int j = 0; j < DEEP; ++j)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const double x = get(v[j], k);
        sum[k & 1] = fma(x, x, sum[k & 1]);
      }
  }
  for (; i < n; i += TPB * N) {
    const Vec<T> v = load_vec(p + i, (long)(n - i));
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const double x = get(v, k);
      sum[k & 1] = fma(x, x, sum[k & 1]);
    }
  }
  return sum[0] + sum[1];
}

__global__ __launch_bounds__(TPB) void clip_squares_kernel(ClipList l, double* sums) {
  __shared__ double part[TPB / 64];
  const int t = find(l, blockIdx.x);
  const size_t begin = (size_t)(blockIdx.x - l.first[t]) * l.piece, all = l.count[t] >> 2, n = all - begin < l.piece ? all - begin : l.piece;
  double s = 0.0;
  OPS_BY_TYPE((int)(l.count[t] & 3), s = squares((const T*)l.p[t] + begin, n));
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// The norm, and behind the sums what the tensors are multiplied by.
constexpr int JOIN = 1024;
__global__ __launch_bounds__(JOIN) void clip_join_kernel(double* sums, unsigned n, double max_norm, float* norm) {
  __shared__ double part[JOIN / 64];
  double s = 0.0;
  for (unsigned i = threadIdx.x; i < n; i += JOIN) s += sums[i];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d, 64);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = 0.0;
  for (int i = 0; i < JOIN / 64; ++i) s += part[i];
  s = sqrt(s);
  if (norm) *norm = (float)s;
  sums[n] = s > max_norm && (float)s < INFINITY ? max_norm / s : 1.0;   // finite as the caller sees it
}

// F: float, or, for a factor that a normal float does not hold (its results may well be such), double.
template <class F, class T>
__device__ __forceinline__ void scaled(const T* p, T* o, size_t n, F f) {
  constexpr int N = Vec<T>::N, DEEP = 4;
  const auto times = [&](const Vec<T>& v) {
    float x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = (float)(get(v, k) * f);
    return f == (F)1 ? v : pack<T>(x);
  };
  size_t i = threadIdx.x * N;
  for (; i + (DEEP - 1) * TPB * N + N <= n; i += DEEP * TPB * N) {
    Vec<T> v[DEEP];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) v[j] = load_vec(p + i + (size_t)j * TPB * N, N);
#pragma unroll
    for (int j = 0; j < DEEP; ++j) store_vec(o + i + (size_t)j * TPB * N, times(v[j]), N);
  }
  for (; i < n; i += TPB * N) store_vec(o + i, times(load_vec(p + i, (long)(n - i))), (long)(n - i));
}

__global__ __launch_bounds__(TPB) void clip_scale_kernel(ClipList l, const double* factor) {
  const unsigned piece = gridDim.x - 1 - blockIdx.x;
  const int t = find(l, piece);
  const float f = (float)*factor;
  if (!l.out[t] || (f == 1.f && l.out[t] == l.p[t])) return;
  const size_t begin = (size_t)(piece - l.first[t]) * l.piece, all = l.count[t] >> 2, n = all - begin < l.piece ? all - begin : l.piece;
  if (f >= FLT_MIN || *factor == 0.0) {
    OPS_BY_TYPE((int)(l.count[t] & 3), scaled((const T*)l.p[t] + begin, (T*)l.out[t] + begin, n, f));
  } else {
    OPS_BY_TYPE((int)(l.count[t] & 3), scaled((const T*)l.p[t] + begin, (T*)l.out[t] + begin, n, *factor));
  }
}

// Elements of a piece: enough for a workgroup's time on them to hide its beginning, fewer where a call is a latency, more where the pieces would
// be too many to add up.
size_t piece_of(size_t total) {
  size_t p = total < (size_t)1 << 22 ? 4096 : 16384;
  while (total / p > 65536) p *= 2;
  return p;
}

size_t total_of(size_t n, const ClipTensor* t) {
  size_t total = 0;
  for (size_t i = 0; i < n; ++i) total += t[i].n;
  return total;
}

size_t pieces_of(size_t n, const ClipTensor* t, size_t piece) {
  size_t pieces = 0;
  for (size_t i = 0; i < n; ++i) pieces += (t[i].n + piece - 1) / piece;
  return pieces;
}

}  // namespace

extern "C" size_t amp_clip_workspace_bytes(size_t n, const ClipTensor* t) { return (pieces_of(n, t, piece_of(total_of(n, t))) + 2) * sizeof(double); }

extern "C" hipError_t amp_clip_launch(size_t n, const ClipTensor* t, double max_norm, float* norm, void* workspace, hipStream_t stream) {
  double* sums = (double*)workspace;
  const size_t piece = piece_of(total_of(n, t)), pieces = pieces_of(n, t, piece);
  static_assert(sizeof(ClipList) <= 4000, "a launch has 4 KB of arguments");
  ClipList l;
  l.piece = piece;
  // the tensors from `from` on (or down to 0) that fit one launch; returns the first of the next
  const auto gather = [&](size_t from, size_t to) {
    l.n = 0, l.first[0] = 0;
    for (size_t i = from; i < to; ++i) {
      if (!t[i].n) continue;
      l.p[l.n] = t[i].p, l.out[l.n] = t[i].out, l.count[l.n] = t[i].n << 2 | (size_t)t[i].dtype;
      l.first[l.n + 1] = l.first[l.n] + (unsigned)((t[i].n + piece - 1) / piece);
      ++l.n;
    }
  };
  hipError_t e = hipSuccess;
  size_t base = 0;
  bool any = false;
  for (size_t i = 0; i < n && e == hipSuccess; i += CLIP_LIST) {
    gather(i, i + CLIP_LIST < n ? i + CLIP_LIST : n);
    if (!l.n) continue;
    for (int k = 0; k < l.n; ++k) any = any || l.out[k];
    e = launch(clip_squares_kernel, dim3(l.first[l.n]), dim3(TPB), 0, stream, l, sums + base);
    base += l.first[l.n];
  }
  if (e == hipSuccess) e = launch(clip_join_kernel, dim3(1), dim3(JOIN), 0, stream, sums, (unsigned)pieces, max_norm, norm);
  if (!any) return e;
  for (size_t end = n; end > 0 && e == hipSuccess;) {
    const size_t begin = (end - 1) / CLIP_LIST * CLIP_LIST;
    gather(begin, end);
    end = begin;
    if (l.n) e = launch(clip_scale_kernel, dim3(l.first[l.n]), dim3(TPB), 0, stream, l, sums + pieces);
  }
  return e;
}
