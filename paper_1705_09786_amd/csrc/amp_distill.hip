// Distillation from a teacher's top logits: loss and gradient (include/amp.h has the formulas).
//
// Bound by HBM: a workgroup keeps a row of logits in its registers from the sum of the exponentials to the gradient, so that each
// logit is read once and its gradient written once, at the rate of a copy for rows that leave room for several workgroups on a compute
// unit (8,192 x 32,000 bf16: 203 us, 5.2 TB/s).  A workgroup has one row: its registers are free for the next one's loads as soon as
// its stores are on their way (workgroups that stay and fetch the next row while they write one took 330 us there, waiting for their
// own stores in front of the loads behind them).
#include "amp_ops.hip.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A softmax's terms are 2^(x scale - m), with m a multiple of scale (the maximum's) or, EXACT, 2^((x - m) scale) with m a logit.  The
// first is one fma and rounds m once for all terms, which the quotient of two sums does not see.  It is no number where a
// scaled logit passes the type's range; rows whose sum it leaves at 0, infinite or no number (all logits at the type's lowest value,
// logits that are infinite or NaN) are done again by the second, which has the plain formula's result.
template <bool EXACT>
__device__ __forceinline__ float exponent(float x, float m, float scale) { return EXACT ? (x - m) * scale : fmaf(x, scale, -m); }
template <bool EXACT>
__device__ __forceinline__ float term(float x, float m, float scale) { return __builtin_amdgcn_exp2f(exponent<EXACT>(x, m, scale)); }
__device__ __forceinline__ float origin(float m) { return m == -INFINITY ? 0.f : m; }
// What a sum over terms of m is worth where the terms are those of top.
template <bool EXACT>
__device__ __forceinline__ float rescale(float m, float top, float scale) {
  return __builtin_amdgcn_exp2f(EXACT ? (m - origin(top)) * scale : m - origin(top));
}

// N more logits, those that `in` says, to a maximum and a sum.
template <bool EXACT, int N, class F>
__device__ __forceinline__ void add_terms(float& m, float& s, const float (&y)[N], F in, float scale) {
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; ++k) top = fmaxf(top, in(k) ? y[k] : -INFINITY);
  top = fmaxf(m, EXACT ? top : fmaxf(top, -1e30f) * scale);
  const float o = EXACT ? origin(top) : top;
  s *= rescale<EXACT>(m, top, scale);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float e = term<EXACT>(y[k], o, scale);
    s += in(k) ? e : 0.f;
  }
  m = top;
}

// Maximum and sum over W lanes; of no terms -infinity and 0.
template <int W, bool EXACT>
__device__ __forceinline__ void group_join(float& m, float& s, float scale) {
  const float top = group_max<W>(m);
  s = group_sum<W>(s * rescale<EXACT>(m, top, scale));
  m = top;
}

__device__ __forceinline__ float teacher_at(const DistillArgs& a, size_t i) {
  return a.teacher_dtype == 0 ? ((const float*)a.teacher)[i] : a.teacher_dtype == 1 ? widen(((const bf16*)a.teacher)[i]) : widen(((const f16*)a.teacher)[i]);
}
// The class of an entry, -1 where it is none.
__device__ __forceinline__ int class_at(const DistillArgs& a, size_t i) {
  const long c = a.index_bytes == 8 ? ((const long*)a.index)[i] : (long)((const int*)a.index)[i];
  return c >= 0 && c < (long)a.classes ? (int)c : -1;
}

template <int TPB>
struct Shared {
  float p[OPS_MAX_TOP], at[OPS_MAX_TOP];   // an entry's probability, the student's logit at its class
  alignas(16) int cls[OPS_MAX_TOP];        // its class, -1 = left out; as many as `top` in fours
  float m[TPB / 64], s[TPB / 64], tm[TPB / 64], ts[TPB / 64], loss[TPB / 64];
};

// A thread's share of a row's teacher entries.
template <int TPB>
struct Entries {
  static constexpr int PER = OPS_MAX_TOP / TPB;
  float y[PER], x[PER];
  int cls[PER];
  __device__ void fetch(const DistillArgs& a, size_t r) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int k = threadIdx.x + i * TPB;
      cls[i] = -1;
      if (k < a.top) {
        y[i] = teacher_at(a, r * a.teacher_stride + k);
        cls[i] = class_at(a, r * a.index_stride + k);
        if (y[i] == -INFINITY) cls[i] = -1;
      }
    }
  }
  template <class T>
  __device__ void gather(const T* row) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (cls[i] >= 0) x[i] = widen(row[cls[i]]);
  }
};

// From the threads' maxima and sums to the workgroup's.
template <int TPB, bool EXACT>
__device__ __forceinline__ void row_join(float& m, float& s, const Entries<TPB>& e, float& tm, float& ts, float scale, Shared<TPB>& t) {
  constexpr int NW = TPB / 64;
  tm = -INFINITY, ts = 0.f;
#pragma unroll
  for (int i = 0; i < Entries<TPB>::PER; ++i)
    if (e.cls[i] >= 0) tm = fmaxf(tm, e.y[i]);
#pragma unroll
  for (int i = 0; i < Entries<TPB>::PER; ++i)
    if (e.cls[i] >= 0) ts += term<true>(e.y[i], origin(tm), scale);
  group_join<64, EXACT>(m, s, scale);
  group_join<64, true>(tm, ts, scale);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (lane == 0) t.m[wave] = m, t.s[wave] = s, t.tm[wave] = tm, t.ts[wave] = ts;
  __syncthreads();
  m = t.m[lane % NW], s = t.s[lane % NW], tm = t.tm[lane % NW], ts = t.ts[lane % NW];
  group_join<NW, EXACT>(m, s, scale);
  group_join<NW, true>(tm, ts, scale);
}

// The threads' parts of sum p (log p - log q), in units of log 2, and the entries, into LDS.
template <int TPB, bool EXACT>
__device__ __forceinline__ void row_loss(const DistillArgs& a, const Entries<TPB>& e, float m, float s, float tm, float ts, float scale,
                                         Shared<TPB>& t) {
  const float lt = __builtin_amdgcn_logf(ts), ls = __builtin_amdgcn_logf(s), at = EXACT ? origin(m) : m;
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < Entries<TPB>::PER; ++i) {
    const int k = threadIdx.x + i * TPB;
    if (k < (a.top + 3) / 4 * 4) {
      const bool used = e.cls[i] >= 0;
      const float p = used ? term<true>(e.y[i], tm, scale) / ts : 0.f;
      t.cls[k] = e.cls[i];
      t.p[k] = p;
      t.at[k] = used ? e.x[i] : 0.f;
      if (used && p != 0.f) l = fmaf(p, ((e.y[i] - tm) * scale - lt) - (exponent<EXACT>(e.x[i], at, scale) - ls), l);
    }
  }
  l = group_sum<64>(l);
  if ((threadIdx.x & 63) == 0) t.loss[threadIdx.x >> 6] = l;
}

// Behind a barrier: the row's loss, and the gradients of the entries' classes, each by the first entry that names it.
template <int TPB, bool EXACT, class T>
__device__ __forceinline__ void row_entries(const DistillArgs& a, size_t r, float w, float m, float f, float scale, T* dx, const Shared<TPB>& t) {
  if (threadIdx.x == 0 && a.loss) {
    float l = t.loss[0];
#pragma unroll
    for (int i = 1; i < TPB / 64; ++i) l += t.loss[i];
    a.loss[r] = w * a.temperature * a.temperature * LN2 * l;
  }
  if (!dx) return;
  for (int k = threadIdx.x; k < a.top; k += TPB) {
    const int c = t.cls[k];
    if (c < 0) continue;
    float p = 0.f;
    bool first = true;
    for (int j = 0; j < a.top; j += 4) {
      const v4i four = *(const v4i*)(t.cls + j);
      if (four.x == c || four.y == c || four.z == c || four.w == c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (four[i] == c) {
            p += t.p[j + i];
            first = first && j + i >= k;
          }
    }
    if (first) dx[c] = (T)fmaf(f, term<EXACT>(t.at[k], EXACT ? origin(m) : m, scale), -w * a.temperature * p);
  }
}

// A row that is left out: no loss, no gradient.
template <int TPB, class T>
__device__ __forceinline__ void row_left_out(const DistillArgs& a, size_t r, T* dx) {
  constexpr int N = Vec<T>::N;
  if (threadIdx.x == 0 && a.loss) a.loss[r] = 0.f;
  const float zero[N] = {};
  if (dx)
    for (long c = threadIdx.x * N; c < (long)a.classes; c += TPB * N) store_vec(dx + c, pack<T>(zero), (long)a.classes - c);
}

// A row read twice, for the sum and for the gradient, with EXACT terms.
template <int TPB, class T>
__device__ __forceinline__ void row_twice(const DistillArgs& a, size_t r, float w, const Entries<TPB>& e, float scale, const T* x, T* dx,
                                          Shared<TPB>& t) {
  constexpr int N = Vec<T>::N;
  const long classes = (long)a.classes;
  float m = -INFINITY, s = 0.f, tm, ts;
  for (long c = threadIdx.x * N; c < classes; c += TPB * N) {
    const Vec<T> v = load_vec(x + c, classes - c);
    float y[N];
#pragma unroll
    for (int k = 0; k < N; ++k) y[k] = get(v, k);
    add_terms<true>(m, s, y, [&](int k) { return c + k < classes; }, scale);
  }
  row_join<TPB, true>(m, s, e, tm, ts, scale, t);
  if (ts == 0.f) return row_left_out<TPB, T>(a, r, dx);
  row_loss<TPB, true>(a, e, m, s, tm, ts, scale, t);
  const float o = origin(m), f = w * a.temperature / s;
  if (dx)
    for (long c = threadIdx.x * N; c < classes; c += TPB * N) {
      const Vec<T> v = load_vec(x + c, classes - c);
      float out[N];
#pragma unroll
      for (int k = 0; k < N; ++k) out[k] = f * term<true>(get(v, k), o, scale);
      store_vec(dx + c, pack<T>(out), classes - c);
    }
  __syncthreads();
  row_entries<TPB, true, T>(a, r, w, m, f, scale, dx, t);
}

template <class T, int TPB, int NV>
__global__ __launch_bounds__(TPB) void distill_kernel(DistillArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ Shared<TPB> t;
  const float scale = LOG2E / a.temperature;
  const long classes = (long)a.classes, groups = (classes + N - 1) / N;
  // group j of this thread begins at element j TPB N + tid N; the row's last one is moved back to end with the row, and what the group in
  // front of it has as well (skip) does not count twice
  const int last = (int)((groups - 1) / TPB);
  const long g = (long)last * TPB + threadIdx.x;
  const bool mine = g < groups;      // has a group number `last`
  const bool narrow = classes < N;   // a row shorter than a group
  const int skip = mine && !narrow && (g + 1) * N > classes ? (int)((g + 1) * N - classes) : 0;
  const int count = !mine ? 0 : narrow ? (int)classes : N;
  // byte offsets from the row's beginning, which is the same for all
  const unsigned off = threadIdx.x * 16u, off_last = mine ? off + (unsigned)last * (TPB * 16u) - (unsigned)skip * (unsigned)sizeof(T) : 0u;
  const auto at = [&](int j) { return j == last ? off_last : off + (unsigned)j * (TPB * 16u); };
  const size_t r = a.row0 + blockIdx.x;
  const T* x = row_of((const T*)a.logits, r, a.logits_stride);
  T* dx = a.dlogits ? row_of((T*)a.dlogits, r, a.dlogits_stride) : nullptr;
  const float w = a.weight ? a.weight[r] : 1.f;
  if (w == 0.f) return row_left_out<TPB, T>(a, r, dx);
  Entries<TPB> e;
  e.fetch(a, r);
  Vec<T> v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j <= last) v[j] = load_vec((const T*)((const char*)x + at(j)), narrow ? classes : N);
  e.gather(x);
  // this thread's maximum and sum, group by group as they arrive
  float m = -INFINITY, s = 0.f, tm, ts;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j <= last) {
      float y[N];
#pragma unroll
      for (int k = 0; k < N; ++k) y[k] = get(v[j], k);
      if (j < last)
        add_terms<false>(m, s, y, [](int) { return true; }, scale);
      else
        add_terms<false>(m, s, y, [&](int k) { return k >= skip && k < count; }, scale);
    }
  row_join<TPB, false>(m, s, e, tm, ts, scale, t);
  // the same for the whole workgroup
  if (ts == 0.f) return row_left_out<TPB, T>(a, r, dx);
  if (!(s > 0.f && s < INFINITY)) {
    __syncthreads();
    return row_twice<TPB, T>(a, r, w, e, scale, x, dx, t);
  }
  row_loss<TPB, false>(a, e, m, s, tm, ts, scale, t);
  const float f = w * a.temperature / s;
  if (dx)
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j <= last) {
        float out[N];
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = f * term<false>(get(v[j], k), m, scale);
        if (j < last || mine) store_vec((T*)((char*)dx + at(j)), pack<T>(out), narrow ? classes : N);
      }
  __syncthreads();
  row_entries<TPB, false, T>(a, r, w, m, f, scale, dx, t);
}

// Longer rows than the registers hold, above 131,072 classes of 16 bits or 65,536 of 32, are read twice: 2,048 x 152,000 bf16 325 us,
// 1,024 x 128,000 f32 294 us, 1.35 and 1.45 times a copy of what they cannot do without.
constexpr int LONG = 1024;
template <class T>
__global__ __launch_bounds__(LONG) void distill_long_kernel(DistillArgs a) {
  __shared__ Shared<LONG> t;
  const size_t r = a.row0 + blockIdx.x;
  const T* x = row_of((const T*)a.logits, r, a.logits_stride);
  T* dx = a.dlogits ? row_of((T*)a.dlogits, r, a.dlogits_stride) : nullptr;
  const float w = a.weight ? a.weight[r] : 1.f;
  if (w == 0.f) return row_left_out<LONG, T>(a, r, dx);
  Entries<LONG> e;
  e.fetch(a, r);
  e.gather(x);
  row_twice<LONG, T>(a, r, w, e, LOG2E / a.temperature, x, dx, t);
}

// Which workgroup takes a row, by its 16-byte groups: as few threads as hold it in registers with several workgroups on a compute unit.
template <class T>
hipError_t run(const DistillArgs& a, dim3 grid, hipStream_t stream) {
  const size_t groups = (a.classes + Vec<T>::N - 1) / Vec<T>::N;
#define DISTILL(TPB, NV) launch(distill_kernel<T, TPB, NV>, grid, dim3(TPB), 0, stream, a)
  if (groups <= 256) return DISTILL(256, 1);
  if (groups <= 512) return DISTILL(256, 2);
  if (groups <= 1024) return DISTILL(256, 4);
  if (groups <= 2048) return DISTILL(256, 8);
  if (groups <= 4096) return DISTILL(512, 8);
  if (groups <= 8192) return DISTILL(1024, 8);
  if (groups <= 16384) return DISTILL(1024, 16);
  return launch(distill_long_kernel<T>, grid, dim3(LONG), 0, stream, a);
}

}  // namespace

extern "C" size_t amp_distill_workspace_bytes(int, size_t, size_t) { return 0; }

extern "C" hipError_t amp_distill_launch(int dtype, const DistillArgs* a, hipStream_t stream) {
  constexpr size_t MOST = (size_t)1 << 21;   // rows of a launch: 2^32 threads are too many
  DistillArgs b = *a;
  for (b.row0 = 0; b.row0 < a->rows; b.row0 += MOST) {
    const dim3 grid((unsigned)(a->rows - b.row0 < MOST ? a->rows - b.row0 : MOST));
    hipError_t e = hipSuccess;
    OPS_BY_TYPE(dtype, e = run<T>(b, grid, stream));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
