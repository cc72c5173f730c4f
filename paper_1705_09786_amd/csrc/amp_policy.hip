// The clipped policy loss with its gradient, and log-probabilities alone (include/amp.h has the formulas).
//
// Bound by HBM: a workgroup has one row of logits in registers between its sums and the gradient, so that the row is read once, up to 131,072
// classes of 16 bits and 65,536 of 32 (longer ones are read again for their gradient); where there is no gradient, rows of any length go by
// once under a running maximum.  8,192 x 32,000 bf16: 193 us with the gradient (5.4 TB/s), 100 without (5.2); rows that are not aligned to their
// 16-byte groups, 2,048 x 151,111 fp16: 132 without (4.7), 363 with it (3.4 TB/s counted as one reading and one writing; f32 618, 4.0;
// from registers 2,048 x 120,001 bf16 286, 3.4; 60,001 f32 222, 4.4).  A term of the softmax is exp2 of (x - max) times a scale of two
// floats, off by some units of 2^-24. In 32 bits at most 128 terms are added up, a thread's of a row in registers (32 of a row that goes by); sums
// of more, the logarithm and what follows it are in 64, since a ratio next to its limit decides whether the row has a gradient at all.
#include "amp_ops.hip.h"

namespace {

// log2(e) / temperature as high + low, both positive, so that a logit of -infinity is a term of 0.
struct Scale {
  float hi, lo;
  __device__ explicit Scale(double s) {
    hi = (float)s;
    if ((double)hi >= s) hi = __uint_as_float(__float_as_uint(hi) - 1u);
    lo = fmaxf((float)(s - (double)hi), 1e-37f);
  }
  __device__ float term(float x, float m) const {
    const float d = x - m;
    return __builtin_amdgcn_exp2f(fmaf(d, hi, d * lo));
  }
};

// What a row's threads agree on.
struct Row {
  float take, give;   // the gradient at the row's own class; minus what every other term is multiplied by
};

__device__ __forceinline__ long class_at(const PolicyArgs& a, size_t r) {
  const long c = a.index_bytes == 8 ? ((const long*)a.index)[r] : (long)((const int*)a.index)[r];
  return c >= 0 && c < (long)a.classes ? c : -1;
}

// From the logarithm of a row's probability to its loss and gradient: one thread.
__device__ __forceinline__ Row finish(const PolicyArgs& a, size_t r, float w, float x, float m, double sum) {
  Row g = {0.f, 0.f};
  const double lp = ((double)x - (double)m) * a.inverse - log(sum);
  if (a.logprob) a.logprob[r] = (float)lp;
  if (w == 0.f) {
    if (a.loss) a.loss[r] = 0.f;
    return g;
  }
  if (!a.loss && !a.dlogits) return g;
  // without `old` the ratio is 1, whatever the probability: also where that is 0 (a log-probability that is no number goes on)
  const double adv = a.advantage[r], d = a.old ? lp - (double)a.old[r] : isnan(lp) ? lp : 0.0;
  // the ratio counts up to its limit on the side that the advantage asks for (a number that is none goes on)
  const bool limited = adv >= 0.0 ? d > a.log_high : adv < 0.0 && d < a.log_low;
  const double ratio = limited ? (adv >= 0.0 ? a.high : a.low) : exp(d);
  double loss = -adv * ratio, by_lp = limited ? 0.0 : -adv * ratio;
  if (a.reference) {
    const double e = (double)a.reference[r] - lp, grown = expm1(e);
    loss += a.kl * (grown - e);
    by_lp -= a.kl * grown;
  }
  if (a.loss) a.loss[r] = (float)(w * loss);
  const double f = (double)w * by_lp * a.inverse;
  g.take = (float)(-f * expm1(lp));
  g.give = (float)(f / sum);
  return g;
}

// A gradient of zeros; with `all` no loss and no log-probability either.
template <int TPB, class T>
__device__ __forceinline__ void left_out(const PolicyArgs& a, size_t r, T* dx, bool all) {
  constexpr int N = Vec<T>::N;
  if (all && threadIdx.x == 0) {
    if (a.loss) a.loss[r] = 0.f;
    if (a.logprob) a.logprob[r] = 0.f;
  }
  const float zero[N] = {};
  if (dx)
    for (long c = threadIdx.x * N; c < (long)a.classes; c += TPB * N) store_vec(dx + c, pack<T>(zero), (long)a.classes - c);
}

template <int N, class T>
__device__ __forceinline__ void store_gradient(const Scale& scale, const Row& g, float m, const Vec<T, N>& v, long c, long own, T* p, long n) {
  float o[N];
#pragma unroll
  for (int k = 0; k < N; ++k) o[k] = -g.give * scale.term(get(v, k), m);
  if (own >= c && own < c + N)
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (c + k == own) o[k] = g.take;
  store_vec(p, pack<T>(o), n);
}

template <class T, int TPB, int NV>
__global__ __launch_bounds__(TPB) void policy_kernel(PolicyArgs a) {
  constexpr int N = Vec<T>::N, NW = TPB / 64;
  __shared__ float top[NW];
  __shared__ double part[NW];
  __shared__ Row row;
  const Scale scale(a.scale);
  const long classes = (long)a.classes, groups = (classes + N - 1) / N;
  const size_t r = a.row0 + blockIdx.x;
  const T* x = row_of((const T*)a.logits, r, a.logits_stride);
  T* dx = row_of((T*)a.dlogits, r, a.dlogits_stride);
  const float w = a.weight ? a.weight[r] : 1.f;
  const long own = class_at(a, r);
  if ((w == 0.f && !a.logprob) || own < 0) return left_out<TPB, T>(a, r, dx, true);
  // thread l has the groups l, l + TPB, ..; the row's last group is moved back to end with the row, and the elements that the group in front
  // of it has as well count there
  const auto at = [&](int j) { return ((long)j * TPB + threadIdx.x) * N; };
  const auto place = [&](long c) { return c + N <= classes || classes < N ? c : classes - N; };
  Vec<T> v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (at(j) < classes) v[j] = load_vec(x + place(at(j)), classes);
  const float mine = widen(x[own]);
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (at(j) < classes)
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (classes >= N || k < classes) m = fmaxf(m, get(v[j], k));
  m = group_max<64>(m);
  if (threadIdx.x % 64 == 0) top[threadIdx.x / 64] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) m = fmaxf(m, top[i]);
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (at(j) < classes) {
      const int skip = (int)(at(j) - place(at(j)));
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float e = scale.term(get(v[j], k), m);
        s += k >= skip && (classes >= N || k < classes) ? e : 0.f;
      }
    }
  double sum = s;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < NW; ++i) sum += part[i];
    row = finish(a, r, w, mine, m, sum);
  }
  __syncthreads();
  if (w == 0.f) return left_out<TPB, T>(a, r, dx, false);
  const Row g = row;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (at(j) < classes) store_gradient(scale, g, m, v[j], place(at(j)), own, dx + place(at(j)), classes);
}

// Rows under a running maximum: without a gradient, or (GRADIENT) read again for it where registers do not hold them.
template <class T, int TPB, bool GRADIENT>
__global__ __launch_bounds__(TPB) void policy_stream_kernel(PolicyArgs a) {
  constexpr int N = Vec<T>::N, NW = TPB / 64, DEEP = 4;
  __shared__ float top[NW];
  __shared__ double part[NW];
  __shared__ Row row;
  const Scale scale(a.scale);
  const long classes = (long)a.classes;
  const size_t r = a.row0 + blockIdx.x;
  const T* x = row_of((const T*)a.logits, r, a.logits_stride);
  T* dx = GRADIENT ? row_of((T*)a.dlogits, r, a.dlogits_stride) : nullptr;
  const float w = a.weight ? a.weight[r] : 1.f;
  const long own = class_at(a, r);
  if ((w == 0.f && !a.logprob) || own < 0) return left_out<TPB, T>(a, r, dx, true);
  const float mine = widen(x[own]);
  float m = -INFINITY;
  double s = 0.0;   // of any number of terms
  // DEEP groups to the running maximum and its sum; of terms that are all 0 so far (a maximum of -infinity) nothing is left to rescale
  const auto add = [&](const Vec<T>(&v)[DEEP], auto in) {
    float most = m;
#pragma unroll
    for (int j = 0; j < DEEP; ++j)
#pragma unroll
      for (int k = 0; k < N; ++k) most = fmaxf(most, in(j, k) ? get(v[j], k) : -INFINITY);
    const float origin = most == -INFINITY ? 0.f : most;
    if (most > m) s *= m == -INFINITY ? 1.0 : (double)scale.term(m, most);
    m = most;
    float t[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < DEEP; ++j)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float e = scale.term(get(v[j], k), origin);
        t[k & 1] += in(j, k) ? e : 0.f;
      }
    s += (double)(t[0] + t[1]);
  };
  constexpr long TURN = (long)DEEP * TPB * N;
  long c0 = threadIdx.x * N;
  for (; c0 - threadIdx.x * N + TURN <= classes; c0 += TURN) {
    Vec<T> v[DEEP];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) v[j] = load_vec(x + c0 + (long)j * TPB * N, N);
    add(v, [](int, int) { return true; });
  }
  if (c0 - threadIdx.x * N < classes) {
    Vec<T> v[DEEP];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
      const long c = c0 + (long)j * TPB * N;
      v[j] = load_vec(x + (c < classes ? c : 0), classes - c);
    }
    add(v, [&](int j, int k) { return c0 + (long)j * TPB * N + k < classes; });
  }
  const float mt = m;
  m = group_max<64>(m);
  if (threadIdx.x % 64 == 0) top[threadIdx.x / 64] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) m = fmaxf(m, top[i]);
  double sum = mt == -INFINITY ? s : s * scale.term(mt, m);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < NW; ++i) sum += part[i];
    if (m == -INFINITY) sum = NAN;   // no class has a probability
    row = finish(a, r, w, mine, m, sum);
  }
  if (!GRADIENT) return;
  __syncthreads();
  if (w == 0.f) return left_out<TPB, T>(a, r, dx, false);
  const Row g = row;
  for (long c = threadIdx.x * N; c < classes; c += TPB * N) store_gradient(scale, g, m, load_vec(x + c, classes - c), c, own, dx + c, classes - c);
}

// Which workgroup takes a row, by its 16-byte groups: with its gradient as few threads as hold it in registers, so that several rows are on a
// compute unit; without, as few as read it in some turns of four groups (16,384 x 1,000 bf16: 296 us on 1,024 threads, 55 on 256, 19 on
// 64; 8,192 x 32,000: 157, 93; 2,048 x 151,111 fp16: 159, 145 and 139 on 512, as they were compared, with a kernel that takes 132 now).
template <class T>
hipError_t run(const PolicyArgs& a, dim3 grid, hipStream_t stream) {
  const size_t groups = (a.classes + Vec<T>::N - 1) / Vec<T>::N;
#define POLICY(TPB, NV) launch(policy_kernel<T, TPB, NV>, grid, dim3(TPB), 0, stream, a)
#define STREAM(TPB, GRADIENT) launch(policy_stream_kernel<T, TPB, GRADIENT>, grid, dim3(TPB), 0, stream, a)
  if (!a.dlogits) {
    if (groups <= 512) return STREAM(64, false);
    if (groups <= 8192) return STREAM(256, false);
    return STREAM(512, false);
  }
  if (groups <= 64) return POLICY(64, 1);
  if (groups <= 128) return POLICY(64, 2);
  if (groups <= 256) return POLICY(64, 4);
  if (groups <= 512) return POLICY(256, 2);
  if (groups <= 1024) return POLICY(256, 4);
  if (groups <= 2048) return POLICY(256, 8);
  if (groups <= 4096) return POLICY(512, 8);
  if (groups <= 8192) return POLICY(1024, 8);
  if (groups <= 16384) return POLICY(1024, 16);
  return STREAM(1024, true);
}

}  // namespace

extern "C" hipError_t amp_policy_launch(int dtype, const PolicyArgs* a, hipStream_t stream) {
  constexpr size_t MOST = (size_t)1 << 21;   // rows of a launch: 2^32 threads are too many
  PolicyArgs b = *a;
  for (b.row0 = 0; b.row0 < a->rows; b.row0 += MOST) {
    const dim3 grid((unsigned)(a->rows - b.row0 < MOST ? a->rows - b.row0 : MOST));
    hipError_t e = hipSuccess;
    OPS_BY_TYPE(dtype, e = run<T>(b, grid, stream));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
