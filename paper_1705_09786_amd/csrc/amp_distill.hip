// Distillation from a teacher's top logits: loss and gradient (include/amp.h has the formulas).
#include "amp_ops.hip.h"

namespace {

constexpr int TPB = 256, NW = TPB / 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// 2^((x - at) scale).  The difference is formed before it is scaled: a scaled logit may pass the type's range (masks of the
// lowest value) and its rounding, relative to the logit, would be the difference's error.
__device__ __forceinline__ float term(float x, float at, float scale) { return __builtin_amdgcn_exp2f((x - at) * scale); }

// Maximum and sum of the terms so far, either side of a join; -infinity and 0 of nothing.
__device__ __forceinline__ float origin(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float scale) {
  const float top = fmaxf(m, m2), at = origin(top);
  s = s * term(m, at, scale) + s2 * term(m2, at, scale);
  m = top;
}

struct Teacher {
  float p[OPS_MAX_TOP], at[OPS_MAX_TOP];   // probability, the student's logit at the entry's class
  int cls[OPS_MAX_TOP];                    // class, -1 = left out
  float part[2][NW][2];
};

__device__ __forceinline__ float teacher_at(const DistillArgs& a, size_t i) {
  return a.teacher_dtype == 0 ? ((const float*)a.teacher)[i] : a.teacher_dtype == 1 ? widen(((const bf16*)a.teacher)[i]) : widen(((const f16*)a.teacher)[i]);
}

__device__ __forceinline__ void block_join(float& m, float& s, float (*part)[2], float scale) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) join(m, s, __shfl_xor(m, d, 64), __shfl_xor(s, d, 64), scale);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][0] = m, part[threadIdx.x >> 6][1] = s;
  __syncthreads();
  m = part[0][0], s = part[0][1];
#pragma unroll
  for (int w = 1; w < NW; ++w) join(m, s, part[w][0], part[w][1], scale);
}

// One workgroup a row; the logits are read twice, for the sum and for the gradient.
template <class T>
__global__ __launch_bounds__(TPB) void distill_kernel(DistillArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ Teacher t;
  const long classes = (long)a.classes;
  const float scale = LOG2E / a.temperature;
  for (size_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = row_of((const T*)a.logits, r, a.logits_stride);
    T* dx = row_of((T*)a.dlogits, r, a.dlogits_stride);
    const float w = a.weight ? a.weight[r] : 1.f;
    float tm = -INFINITY, ts = 0.f;
    if (w != 0.f) {
      for (int k = threadIdx.x; k < a.top; k += TPB) {
        const size_t i = r * a.index_stride + k;
        const long c = a.index_bytes == 8 ? ((const long*)a.index)[i] : (long)((const int*)a.index)[i];
        const float y = teacher_at(a, r * a.teacher_stride + k);
        const bool used = c >= 0 && c < classes && y != -INFINITY;
        t.cls[k] = used ? (int)c : -1;
        t.p[k] = y;
        t.at[k] = used ? widen(x[c]) : 0.f;
        if (used) join(tm, ts, y, 1.f, scale);
      }
    }
    block_join(tm, ts, t.part[0], scale);
    if (ts == 0.f) {   // no entry, or weight 0: the same for the whole workgroup
      if (threadIdx.x == 0 && a.loss) a.loss[r] = 0.f;
      const float zero[N] = {};
      if (a.dlogits)
        for (long c = threadIdx.x * N; c < classes; c += TPB * N) store_vec(dx + c, pack<T>(zero), classes - c);
      __syncthreads();
      continue;
    }
    float m = -INFINITY, s = 0.f;
    for (long c = threadIdx.x * N; c < classes; c += TPB * N) {
      const Vec<T> v = load_vec(x + c, classes - c);
      float y[N], vm = -INFINITY, vs = 0.f;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        y[k] = c + k < classes ? get(v, k) : -INFINITY;
        vm = fmaxf(vm, y[k]);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) vs += term(y[k], origin(vm), scale);
      join(m, s, vm, vs, scale);
    }
    block_join(m, s, t.part[1], scale);
    const float at = origin(m);
    // loss = sum p (log p - log q), in units of log 2 up to the end
    const float lt = __builtin_amdgcn_logf(ts), ls = __builtin_amdgcn_logf(s);
    float l[1] = {0.f};
    for (int k = threadIdx.x; k < a.top; k += TPB) {
      const bool used = t.cls[k] >= 0;
      const float y = t.p[k], p = used ? term(y, tm, scale) / ts : 0.f;
      t.p[k] = p;
      if (used && p != 0.f) l[0] = fmaf(p, ((y - tm) * scale - lt) - ((t.at[k] - at) * scale - ls), l[0]);
    }
    __shared__ float lpart[NW][1];
    block_sum<NW>(l, lpart);
    if (threadIdx.x == 0 && a.loss) a.loss[r] = w * a.temperature * a.temperature * LN2 * l[0];
    if (a.dlogits) {
      const float f = w * a.temperature / s;
      for (long c = threadIdx.x * N; c < classes; c += TPB * N) {
        const Vec<T> v = load_vec(x + c, classes - c);
        float o[N];
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = f * term(get(v, k), at, scale);
        store_vec(dx + c, pack<T>(o), classes - c);
      }
      __syncthreads();
      // the entries' classes, each by the first entry that names it
      for (int k = threadIdx.x; k < a.top; k += TPB) {
        const int c = t.cls[k];
        if (c < 0) continue;
        float p = 0.f;
        bool first = true;
        for (int j = 0; j < a.top; ++j)
          if (t.cls[j] == c) {
            p += t.p[j];
            first = first && j >= k;
          }
        if (!first) continue;
        const float o = fmaf(f, term(t.at[k], at, scale), -w * a.temperature * p);
        dx[c] = (T)o;
      }
    }
    __syncthreads();
  }
}

}  // namespace

extern "C" size_t amp_distill_workspace_bytes(int, size_t, size_t) { return 0; }

extern "C" hipError_t amp_distill_launch(int dtype, const DistillArgs* a, hipStream_t stream) {
  const dim3 grid((unsigned)(a->rows < 65536 ? a->rows : 65536));
  OPS_BY_TYPE(dtype, return launch(distill_kernel<T>, grid, dim3(TPB), 0, stream, *a));
}
