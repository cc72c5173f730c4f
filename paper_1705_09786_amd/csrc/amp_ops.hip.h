// Device-side building blocks of the operators on whole arrays: element types, 16-byte groups of them at any alignment, reductions.
#pragma once
#include <hip/hip_runtime.h>
#include "amp_ops.h"

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef bf16 v2bf __attribute__((ext_vector_type(2)));
typedef f16 v2h __attribute__((ext_vector_type(2)));

// A group of N elements, 16 bytes (the widest access of a lane) or 8.  Rows start at any element (odd lengths, views): the hardware
// takes such accesses at any address, at a second cache line's cost where one is crossed, so there is no path for unaligned rows.
typedef unsigned v2u __attribute__((ext_vector_type(2)));
template <int WORDS>
struct Words;
template <>
struct Words<4> {
  typedef v4u type;
};
template <>
struct Words<2> {
  typedef v2u type;
};
template <class T, int N_ = 16 / sizeof(T)>
struct Vec {
  static constexpr int N = N_;
  typedef typename Words<N * sizeof(T) / 4>::type U;
  typedef U Any __attribute__((aligned(sizeof(T))));
  U u;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return (float)v; }
__device__ __forceinline__ float widen(f16 v) { return (float)v; }

// The group at p, elements n and later replaced by zeros and not read (n >= N: all of it).
template <int N, class T>
__device__ __forceinline__ Vec<T, N> load_group(const T* p, long n) {
  Vec<T, N> v;
  if (n >= N) {
    v.u = *(const typename Vec<T, N>::Any*)p;
    return v;
  }
  v.u = (typename Vec<T, N>::U)0u;
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < n) {
      if (sizeof(T) == 2)
        v.u[k / 2] |= (unsigned)((const unsigned short*)p)[k] << (16 * (k & 1));
      else
        v.u[k] = ((const unsigned*)p)[k];
    }
  return v;
}
template <class T>
__device__ __forceinline__ Vec<T> load_vec(const T* p, long n) { return load_group<16 / sizeof(T)>(p, n); }

template <class T, int N>
__device__ __forceinline__ void store_vec(T* p, Vec<T, N> v, long n) {
  if (n >= N) {
    *(typename Vec<T, N>::Any*)p = v.u;
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < n) {
      if (sizeof(T) == 2)
        ((unsigned short*)p)[k] = (unsigned short)(v.u[k / 2] >> (16 * (k & 1)));
      else
        ((unsigned*)p)[k] = v.u[k];
    }
}

template <int N>
__device__ __forceinline__ float get(const Vec<float, N>& v, int k) { return __uint_as_float(v.u[k]); }
template <int N>
__device__ __forceinline__ float get(const Vec<bf16, N>& v, int k) {
  const unsigned w = v.u[k / 2];
  return __uint_as_float((k & 1) ? w & 0xffff0000u : w << 16);
}
template <int N>
__device__ __forceinline__ float get(const Vec<f16, N>& v, int k) { return (float)__builtin_bit_cast(v2h, (unsigned)v.u[k / 2])[k & 1]; }

// N floats rounded to the nearest of T, the one rounding of a result.
__device__ __forceinline__ unsigned pack2(float a, float b, bf16) { return __builtin_bit_cast(unsigned, __builtin_convertvector((v2f){a, b}, v2bf)); }
__device__ __forceinline__ unsigned pack2(float a, float b, f16) { return __builtin_bit_cast(unsigned, __builtin_convertvector((v2f){a, b}, v2h)); }
template <class T, int N>
__device__ __forceinline__ Vec<T, N> pack(const float (&f)[N]) {
  Vec<T, N> v;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < N; ++k) v.u[k] = __float_as_uint(f[k]);
  } else {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) v.u[k] = pack2(f[2 * k], f[2 * k + 1], T());
  }
  return v;
}

// Sum and maximum over the W lanes of a lane's aligned group; every lane gets the same bits (both sides of a step add the same two
// values).  A NaN anywhere leaves a NaN in the sum; the maximum passes over it, as fmaxf does.
template <int W>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int d = 1; d < W; d *= 2) v += __shfl_xor(v, d, 64);
  return v;
}
template <int W>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int d = 1; d < W; d *= 2) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}

// Sums of M values over a workgroup of NW waves, the same bits in every thread.  `part` holds NW x M floats; the caller alternates
// between two of them, so that one barrier a call is enough.
template <int NW, int M>
__device__ __forceinline__ void block_sum(float (&v)[M], float (*part)[M]) {
#pragma unroll
  for (int m = 0; m < M; ++m) v[m] = group_sum<64>(v[m]);
  if (NW == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int m = 0; m < M; ++m) part[threadIdx.x >> 6][m] = v[m];
  __syncthreads();
#pragma unroll
  for (int m = 0; m < M; ++m) {
    float s = part[0][m];
#pragma unroll
    for (int w = 1; w < NW; ++w) s += part[w][m];
    v[m] = s;
  }
}

template <class T>
__device__ __forceinline__ T* row_of(T* p, size_t row, size_t stride) { return p + row * stride; }

// Launches a kernel and returns the launch's own status (hipGetLastError would also hand on, and clear, an earlier call's).
template <class P>
struct As {
  typedef P type;
};
template <class... P>
inline hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, unsigned lds, hipStream_t stream, typename As<P>::type... p) {
  void* args[] = {(void*)&p...};
  return hipLaunchKernel((const void*)kernel, grid, block, args, lds, stream);
}

#define OPS_BY_TYPE(dtype, ...)                  \
  switch (dtype) {                               \
    case 0: { typedef float T; __VA_ARGS__; } break;    \
    case 1: { typedef bf16 T; __VA_ARGS__; } break;     \
    default: { typedef f16 T; __VA_ARGS__; } break;     \
  }
