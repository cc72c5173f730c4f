// The gated delta rule, forward, backward and one row at a time (include/amp.h has the formulas).
//
// A sequence is cut into chunks of 32 rows. With G the sum of a chunk's decays up to a row, D_ij = exp(G_i - G_j), S the state in front
// of the chunk and M_ij = D_ij k_i.k_j (i > j), the errors e of all its rows solve (1 + M beta) E = V - e^G K S, and
//   O = scale (e^G Q S + (D o Q K^T) beta E),   S <- e^{G_end} S + (e^{G_end - G} K)^T beta E.
// With N = (1 + M beta)^-1 M that inverse is 1 - N beta, and the one that the backward pass needs, of 1 + beta M, is 1 - beta N: one
// matrix serves both directions. For the backward pass, with X the gradient of beta E and S' that of the state behind the chunk,
//   X = (1 - N^T beta) (P^T dO + e^{G_end - G} K S'),   S <- e^{G_end} S' + (scale e^G Q)^T dO - (e^G K)^T beta X,
// where P = scale D o Q K^T; every other gradient follows from E, X and the states at a chunk's two ends, for chunks of any length.
//
// Kernels: (1) the plan, the blocks of 64 rows in front of every sequence; (2) per block and head, N and P of its two chunks; (3) the
// chain, a workgroup for each sequence and head, whose waves have 16 columns of the state each in registers for the whole sequence: a
// state is both result and operand of the matrix instructions in the layout that it has there, so that nothing but K, Q, N and P passes
// through LDS; (4) backward, the chain the other way; and (5) per block, the gradients.
//
// Products run on the bf16 matrix instructions, whose operands hold 8 bits: a number is the sum of up to three of them (24 bits, as in 32-bit
// arithmetic; an input in bf16 is one, in fp16 two), and of a product's partial products those are taken that reach 2^-24 of it. That is
// three instructions for an input in bf16 with a state, six for a state with a state, each of 16 times the rate of the 32-bit ones.
#include "amp_ops.hip.h"

namespace {

constexpr int C = DELTA_CHUNK, B = DELTA_BLOCK;
typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

template <class T>
struct In {
  static constexpr int P = sizeof(T) == 4 ? 3 : 2;   // parts of an input
};
template <>
struct In<bf16> {
  static constexpr int P = 1;
};

// ------------------------------------------------------------------ operands of the matrix instruction
// A lane's eight elements along the contraction, in parts. Operands meet in the order that the elements have here, whatever numbers
// they stand for: where one side is a product's result (rows 4 (lane / 16) + i of a tile of 16), both have the rows of two tiles so.
template <int P>
struct Frag {
  v4u p[P];
};

template <int P>
__device__ __forceinline__ void split2(float a, float b, unsigned (&u)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    u[i] = pack2(a, b, bf16());
    if (i + 1 < P) {
      a -= __uint_as_float(u[i] << 16);
      b -= __uint_as_float(u[i] & 0xffff0000u);
    }
  }
}
template <int P>
__device__ __forceinline__ Frag<P> split8(const float (&x)[8]) {
  Frag<P> f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    unsigned u[P];
    split2<P>(x[2 * k], x[2 * k + 1], u);
#pragma unroll
    for (int i = 0; i < P; ++i) f.p[i][k] = u[i];
  }
  return f;
}

// c + a b, of the partial products i, j those with i + j < ORDER, the smallest first.
template <int ORDER, int PA, int PB>
__device__ __forceinline__ v4f mma(const Frag<PA>& a, const Frag<PB>& b, v4f c) {
#pragma unroll
  for (int s = ORDER - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i)
      if (s - i >= 0 && s - i < PB)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a.p[i]), __builtin_bit_cast(v8bf, b.p[s - i]), c, 0, 0, 0);
  return c;
}

// Matrices in LDS: parts, rows, LD elements a row. Their columns lie in fours; of 32 columns the fours 0, 4, 1, 5, 2, 6, 3, 7 are next to
// each other (`place`), so that a lane's eight along a row, columns 4 q .. and 16 + 4 q .., are 16 bytes.
__device__ __forceinline__ int place(int four) { return (four / 8) * 32 + (four % 4) * 8 + (four / 4 % 2) * 4; }

template <int P, int ROWS, int LD>
struct Matrix {
  alignas(16) bf16 at[P][ROWS][LD];
  // the operand whose lane has row `row`, contracted over the columns 32 f ..
  __device__ __forceinline__ Frag<P> along_row(int row, int f) const {
    Frag<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i) r.p[i] = *(const v4u*)&at[i][row][f * 32 + (threadIdx.x % 64 / 16) * 8];
    return r;
  }
  // the operand whose lane has column 16 tile + lane % 16, contracted over the rows row0 ..: read transposed, four rows of 16 columns
  // to 16 lanes
  __device__ __forceinline__ Frag<P> down(int tile, int row0) const {
    const int lane = threadIdx.x % 64, q = lane / 16, row = row0 + 4 * q + lane % 16 / 4, col = place(4 * tile + lane % 4);
    Frag<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const v2u lo = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)&at[i][row][col]));
      const v2u hi = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)&at[i][row + 16][col]));
      r.p[i] = (v4u){lo.x, lo.y, hi.x, hi.y};
    }
    return r;
  }
  // four columns from 4 `four` on
  __device__ __forceinline__ void put(int row, int four, const v2u (&u)[P]) {
#pragma unroll
    for (int i = 0; i < P; ++i) *(v2u*)&at[i][row][place(four)] = u[i];
  }
};

template <int P>
__device__ __forceinline__ void split4(const float (&x)[4], v2u (&u)[P]) {
  unsigned a[P], b[P];
  split2<P>(x[0], x[1], a);
  split2<P>(x[2], x[3], b);
#pragma unroll
  for (int i = 0; i < P; ++i) u[i] = (v2u){a[i], b[i]};
}
__device__ __forceinline__ void parts4(const Vec<bf16, 4>& v, v2u (&u)[1]) { u[0] = v.u; }
template <class T, int P>
__device__ __forceinline__ void parts4(const Vec<T, 4>& v, v2u (&u)[P]) {
  const float x[4] = {get(v, 0), get(v, 1), get(v, 2), get(v, 3)};
  split4<P>(x, u);
}

// ------------------------------------------------------------------ where things are
struct Block {
  long row;      // its first row
  int count;     // its rows
  size_t index;
};

__device__ __forceinline__ long bound_at(const DeltaArgs& a, const void* p, size_t s) {
  return a.index_bytes == 8 ? ((const long*)p)[s] : (long)((const int*)p)[s];
}
// A sequence's rows, within the arrays whatever its bounds say.
__device__ __forceinline__ void span(const DeltaArgs& a, size_t s, long& b, long& e) {
  b = 0, e = (long)a.rows;
  if (!a.begin) return;
  const long x = bound_at(a, a.begin, s), y = bound_at(a, a.end, s);
  b = x < 0 ? 0 : x > e ? e : x;
  e = y < b ? b : y > e ? e : y;
}
// Blocks in front of a sequence, at most the workspace's number of them.
__device__ __forceinline__ long first_block(const DeltaArgs& a, size_t s) { return a.begin ? a.first[s] : s ? (long)a.blocks : 0; }

__device__ __forceinline__ bool find_block(const DeltaArgs& a, size_t index, Block& w) {
  size_t lo = 0, hi = a.n_seq;   // first[lo] <= index < first[hi]
  if ((long)index >= first_block(a, hi)) return false;
  while (hi - lo > 1) {
    const size_t mid = (lo + hi) / 2;
    (first_block(a, mid) <= (long)index ? lo : hi) = mid;
  }
  long b, e;
  span(a, lo, b, e);
  w.row = b + ((long)index - first_block(a, lo)) * B;
  w.count = e - w.row < B ? (int)(e - w.row) : B;
  w.index = index;
  return w.count > 0;
}

// N and P of a chunk, the sums of decays of a block's two chunks (in 64 bits: differences of far sums decide about near rows).
__device__ __forceinline__ float* matrices_of(const DeltaArgs& a, size_t block, int h, int chunk) {
  return a.matrices + ((block * a.heads + h) * 2 + chunk) * (2 * C * C);
}
__device__ __forceinline__ double* sums_of(const DeltaArgs& a, size_t block, int h) { return a.sums + (block * a.heads + h) * B; }
__device__ __forceinline__ size_t state_at(const DeltaArgs& a, size_t index, int h) { return (index * a.heads + h) * ((size_t)a.dk * a.dv); }

// ------------------------------------------------------------------ plan
constexpr int PLAN = 1024;
__global__ __launch_bounds__(PLAN) void delta_plan_kernel(DeltaArgs a) {
  __shared__ long part[PLAN / 64];
  long base = 0;
  for (size_t s0 = 0; s0 < a.n_seq; s0 += PLAN) {
    const size_t s = s0 + threadIdx.x;
    long b = 0, e = 0;
    if (s < a.n_seq) span(a, s, b, e);
    const long mine = (e - b + B - 1) / B;
    long sum = mine;
    for (int d = 1; d < 64; d *= 2) {
      const long up = __shfl_up(sum, d, 64);
      if ((int)(threadIdx.x & 63) >= d) sum += up;
    }
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    long front = base;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) front += part[w];
    const long at = front + sum - mine;
    if (s < a.n_seq) a.first[s] = at < (long)a.blocks ? (int)at : (int)a.blocks;
    for (int w = threadIdx.x >> 6; w < PLAN / 64; ++w) front += part[w];
    base = front;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.first[a.n_seq] = base < (long)a.blocks ? (int)base : (int)a.blocks;
}

// Rows of no sequence: a wave to a row, zeros in every output.
__global__ __launch_bounds__(256) void delta_zero_kernel(DeltaArgs a) {
  for (size_t row = (size_t)blockIdx.x * 4 + threadIdx.x / 64; row < a.rows; row += (size_t)gridDim.x * 4) {
    size_t lo = 0, hi = a.n_seq;   // the last sequence that begins at or in front of the row, if any
    while (lo < hi) {
      const size_t mid = (lo + hi) / 2;
      if (bound_at(a, a.begin, mid) <= (long)row) lo = mid + 1;
      else hi = mid;
    }
    if (lo) {
      long b, e;
      span(a, lo - 1, b, e);
      if ((long)row < e) continue;
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      if (!a.zero[k].p) continue;
      char* p = (char*)a.zero[k].p + row * a.zero[k].stride;
      for (size_t i = threadIdx.x % 64; i < a.zero[k].halves; i += 64) ((unsigned short*)p)[i] = 0;
    }
  }
}

// ------------------------------------------------------------------ per block and head: N, P and the sums of decays
template <class T, int KT>
__global__ __launch_bounds__(256) void delta_prepare_kernel(DeltaArgs a) {
  constexpr int P = In<T>::P, LD = KT * 32 + 8;
  __shared__ Matrix<P, B, LD> k, q;
  __shared__ float mat[2][2][C][C + 4];   // chunk, K K^T or Q K^T
  __shared__ double g[B];
  __shared__ float beta[B];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads);
  Block w;
  if (!find_block(a, blockIdx.x / a.heads, w)) return;
  const T* K = row_of((const T*)a.k, w.row, a.k_stride) + (size_t)hk * a.dk;
  const T* Q = row_of((const T*)a.q, w.row, a.q_stride) + (size_t)hk * a.dk;
  constexpr int UNITS = B * KT * 8;
#pragma unroll
  for (int j = 0; j < UNITS / 256; ++j) {
    const int u = threadIdx.x + j * 256, row = u / (KT * 8), four = u % (KT * 8);
    const long n = row < w.count ? a.dk - four * 4 : 0;
    v2u x[P];
    parts4(load_group<4>(K + (row < w.count ? row : 0) * a.k_stride + (n > 0 ? four * 4 : 0), n), x);
    k.put(row, four, x);
    parts4(load_group<4>(Q + (row < w.count ? row : 0) * a.q_stride + (n > 0 ? four * 4 : 0), n), x);
    q.put(row, four, x);
  }
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  if (wave == 0) {
    float d = 0.f, bt = 0.f;
    if (lane < w.count) {
      d = a.decay[(w.row + lane) * a.decay_stride + h];
      bt = a.beta[(w.row + lane) * a.beta_stride + h];
    }
    // e^-1000 is 0; -infinity, which forgets everything as well, would leave no differences
    double sum = d < -1000.f ? -1000.0 : (double)d;
#pragma unroll
    for (int s = 1; s < C; s *= 2) {
      const double up = __shfl_up(sum, s, C);
      if (lane % C >= s) sum += up;
    }
    g[lane] = sum;
    beta[lane] = bt;
    sums_of(a, w.index, h)[lane] = sum;
  }
  __syncthreads();
  {   // a wave to each product of each chunk: its three tiles that have elements on or below the diagonal
    const int chunk = wave / 2, r0 = chunk * C, c = lane % 16;
    const Matrix<P, B, LD>& left = wave % 2 ? q : k;
    v4f acc[3] = {};
#pragma unroll
    for (int f = 0; f < KT; ++f) {
      const Frag<P> a0 = left.along_row(r0 + c, f), a1 = left.along_row(r0 + 16 + c, f);
      const Frag<P> b0 = k.along_row(r0 + c, f), b1 = k.along_row(r0 + 16 + c, f);
      acc[0] = mma<3>(a0, b0, acc[0]);
      acc[1] = mma<3>(a1, b0, acc[1]);
      acc[2] = mma<3>(a1, b1, acc[2]);
    }
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) mat[chunk][wave % 2][(t ? 16 : 0) + 4 * (lane / 16) + i][(t == 2 ? 16 : 0) + c] = acc[t][i];
  }
  __syncthreads();
  // the decays: P is finished, M beta takes M's place
#pragma unroll
  for (int j = 0; j < 2 * C * C / 256; ++j) {
    const int e = threadIdx.x + j * 256, chunk = e / (C * C), r = e / C % C, c = e % C;
    const float d = r >= c ? expf((float)(g[chunk * C + r] - g[chunk * C + c])) : 0.f;
    matrices_of(a, w.index, h, chunk)[C * C + r * C + c] = r >= c ? a.scale * d * mat[chunk][1][r][c] : 0.f;
    mat[chunk][1][r][c] = r > c ? d * mat[chunk][0][r][c] : 0.f;
    mat[chunk][0][r][c] = r > c ? d * mat[chunk][0][r][c] * beta[chunk * C + c] : 0.f;
  }
  __syncthreads();
  // N = M - (M beta) N, row after row, a lane to a column
  if (wave == 0) {
    const int chunk = lane / C, c = lane % C;
    float n[C];
    float* out = matrices_of(a, w.index, h, chunk);
#pragma unroll
    for (int r = 0; r < C; ++r) {
      float s[4] = {mat[chunk][1][r][c], 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < r; ++m) s[m % 4] = fmaf(-mat[chunk][0][r][m], n[m], s[m % 4]);
      n[r] = (s[0] + s[1]) + (s[2] + s[3]);
      out[r * C + c] = n[r];
    }
  }
}

// ------------------------------------------------------------------ the chain over a sequence's chunks
// What a chunk's waves share, on its way from memory and in LDS.
template <class T, int KT, int W, int PN>
struct Chunk {
  static constexpr int P = In<T>::P, LD = KT * 32 + 8, UNITS = C * KT * 8, PER = (UNITS + 64 * W - 1) / (64 * W), PAIR = 2 * C * C / 4 / (64 * W);
  struct Shared {
    Matrix<P, C, LD> k, q;
    Matrix<3, C, C + 8> n;
    Matrix<PN, C, C + 8> p;
    float beta[C], grow[C], rest[C], whole;
  };
  Vec<T, 4> k[PER], q[PER];
  Vec<float, 4> pair[PAIR];
  double g, end;
  float beta;
  __device__ __forceinline__ void fetch(const DeltaArgs& a, long row, int count, size_t block, int half, int h, int hk) {
    const T* K = row_of((const T*)a.k, row, a.k_stride) + (size_t)hk * a.dk;
    const T* Q = row_of((const T*)a.q, row, a.q_stride) + (size_t)hk * a.dk;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int u = threadIdx.x + j * 64 * W, r = u / (KT * 8), four = u % (KT * 8);
      const long n = r < count ? a.dk - four * 4 : 0;
      const int rr = r < count ? r : 0, cc = n > 0 ? four * 4 : 0;
      k[j] = load_group<4>(K + rr * a.k_stride + cc, n);
      q[j] = load_group<4>(Q + rr * a.q_stride + cc, n);
    }
    const float* m = matrices_of(a, block, h, half);
#pragma unroll
    for (int j = 0; j < PAIR; ++j) pair[j] = load_vec(m + (threadIdx.x + j * 64 * W) * 4, 4);
    const double* sums = sums_of(a, block, h) + half * C;
    g = sums[threadIdx.x % C], end = sums[C - 1];
    const int r = threadIdx.x % C;
    beta = r < count ? a.beta[(row + r) * a.beta_stride + h] : 0.f;
  }
  __device__ __forceinline__ void put(Shared& s) const {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int u = threadIdx.x + j * 64 * W;
      if (UNITS % (64 * W) && u >= UNITS) continue;
      v2u x[P];
      parts4(k[j], x);
      s.k.put(u / (KT * 8), u % (KT * 8), x);
      parts4(q[j], x);
      s.q.put(u / (KT * 8), u % (KT * 8), x);
    }
#pragma unroll
    for (int j = 0; j < PAIR; ++j) {
      const int u = threadIdx.x + j * 64 * W, r = u % (C * C / 4) / (C / 4), four = u % (C / 4);
      const float x[4] = {get(pair[j], 0), get(pair[j], 1), get(pair[j], 2), get(pair[j], 3)};
      if (u < C * C / 4) {
        v2u y[3];
        split4<3>(x, y);
        s.n.put(r, four, y);
      } else {
        v2u y[PN];
        split4<PN>(x, y);
        s.p.put(r, four, y);
      }
    }
    if (threadIdx.x < C) {
      s.beta[threadIdx.x] = beta;
      s.grow[threadIdx.x] = expf((float)g);
      s.rest[threadIdx.x] = expf((float)(end - g));
      if (threadIdx.x == 0) s.whole = expf((float)end);
    }
  }
};

// Eight of a wave's values in a chunk: rows 4 (lane / 16) + i of its two tiles, column lane % 16 of the wave's.
__device__ __forceinline__ int chunk_row(int k) { return (k / 4) * 16 + 4 * (threadIdx.x % 64 / 16) + k % 4; }

template <class T>
struct Rows8 {
  T v[8];
  __device__ __forceinline__ void fetch(const T* p, size_t stride, int count, bool column) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = (T)0.f;
      if (column && chunk_row(k) < count) v[k] = p[chunk_row(k) * stride];
    }
  }
};

// A state's 16 columns in a wave: element i of tile m is row 16 m + 4 (lane / 16) + i.
template <int KT>
struct State {
  v4f t[2 * KT];
  __device__ __forceinline__ void load(const DeltaArgs& a, const float* p, int col) {
    const int r0 = 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) t[m][i] = p && col < a.dv && 16 * m + r0 + i < a.dk ? p[(size_t)(16 * m + r0 + i) * a.dv + col] : 0.f;
  }
  __device__ __forceinline__ void store(const DeltaArgs& a, float* p, int col) const {
    const int r0 = 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col < a.dv && 16 * m + r0 + i < a.dk) p[(size_t)(16 * m + r0 + i) * a.dv + col] = t[m][i];
  }
  __device__ __forceinline__ Frag<3> operand(int f) const {
    const float x[8] = {t[2 * f][0], t[2 * f][1], t[2 * f][2], t[2 * f][3], t[2 * f + 1][0], t[2 * f + 1][1], t[2 * f + 1][2], t[2 * f + 1][3]};
    return split8<3>(x);
  }
};

template <class T, int KT, int W>
__global__ __launch_bounds__(64 * W) void delta_forward_kernel(DeltaArgs a) {
  constexpr int PO = sizeof(T) == 2 ? 2 : 3;   // o is rounded to 16 bits: two parts leave 2^-16 of its terms
  typedef Chunk<T, KT, W, PO> Ck;
  __shared__ typename Ck::Shared sh[2];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads);
  const size_t s = blockIdx.x / a.heads;
  const int lane = threadIdx.x % 64, c16 = lane % 16, q = lane / 16, c0 = (blockIdx.y * W + threadIdx.x / 64) * 16, col = c0 + c16;
  long b, e;
  span(a, s, b, e);
  const long first = first_block(a, s), all = first_block(a, s + 1);
  if (e > b + (all - first) * B) e = b + (all - first) * B;
  State<KT> S;
  S.load(a, a.h0 ? a.h0 + state_at(a, s, h) : nullptr, col);
  const T* V = (const T*)a.v + (size_t)h * a.dv + col;
  const int chunks = (int)((e - b + C - 1) / C);
  const auto rows_in = [&](int c) { return e - b - (long)c * C < C ? (int)(e - b - (long)c * C) : C; };
  Ck next;
  Rows8<T> vnext;
  const auto fetch = [&](int c) {
    const long row = b + (long)c * C;
    next.fetch(a, row, rows_in(c), (size_t)(first + c / 2), c % 2, h, hk);
    vnext.fetch(V + row * a.v_stride, a.v_stride, rows_in(c), col < a.dv);
  };
  if (chunks > 0) {
    fetch(0);
    next.put(sh[0]);
  }
  Rows8<T> v = vnext;
  __syncthreads();
  for (int c = 0; c < chunks; ++c) {
    const typename Ck::Shared& t = sh[c & 1];
    const long row = b + (long)c * C;
    const int count = rows_in(c);
    if (c + 1 < chunks) fetch(c + 1);
    if (c0 < a.dv) {
      if (a.carry && c % 2 == 0) S.store(a, a.carry + a.carry_states + state_at(a, (size_t)(first + c / 2), h), col);
      Frag<3> op[KT];
#pragma unroll
      for (int f = 0; f < KT; ++f) op[f] = S.operand(f);
      v4f ks[2] = {}, oq[2] = {};
#pragma unroll
      for (int f = 0; f < KT; ++f)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          ks[r] = mma<3>(t.k.along_row(16 * r + c16, f), op[f], ks[r]);
          oq[r] = mma<PO>(op[f], t.q.along_row(16 * r + c16, f), oq[r]);
        }
      float x[8], y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = widen(v.v[k]) - t.grow[chunk_row(k)] * ks[k / 4][k % 4];
        y[k] = t.beta[chunk_row(k)] * x[k];
      }
      const Frag<3> rb = split8<3>(y);
      v4f nr[2] = {};
#pragma unroll
      for (int r = 0; r < 2; ++r) nr[r] = mma<3>(t.n.along_row(16 * r + c16, 0), rb, nr[r]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] -= nr[k / 4][k % 4];
        if (a.carry && col < a.dv && chunk_row(k) < count) a.carry[(row + chunk_row(k)) * ((size_t)a.heads * a.dv) + (size_t)h * a.dv + col] = x[k];
        x[k] *= t.beta[chunk_row(k)];
        y[k] = t.rest[chunk_row(k)] * x[k];
      }
      const Frag<3> up = split8<3>(y);
      const float whole = t.whole;
#pragma unroll
      for (int m = 0; m < 2 * KT; ++m) S.t[m] = mma<3>(t.k.down(m, 0), up, S.t[m] * whole);
      if (a.o) {
        const Frag<PO> vo = split8<PO>(x);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          oq[r] = mma<PO>(vo, t.p.along_row(16 * r + c16, 0), oq[r] * (t.grow[16 * r + c16] * a.scale));
          if (16 * r + c16 < count) {
            const float o[4] = {oq[r][0], oq[r][1], oq[r][2], oq[r][3]};
            store_vec((T*)a.o + (row + 16 * r + c16) * a.o_stride + (size_t)h * a.dv + c0 + 4 * q, pack<T>(o), a.dv - c0 - 4 * q);
          }
        }
      }
    }
    if (c + 1 < chunks) {
      next.put(sh[(c + 1) & 1]);
      v = vnext;
    }
    __syncthreads();
  }
  if (a.last) S.store(a, a.last + state_at(a, s, h), col);
}

template <class T, int KT, int W>
__global__ __launch_bounds__(64 * W) void delta_backward_kernel(DeltaArgs a) {
  typedef Chunk<T, KT, W, 3> Ck;
  constexpr int P = In<T>::P;
  __shared__ typename Ck::Shared sh[2];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads);
  const size_t s = blockIdx.x / a.heads;
  const int lane = threadIdx.x % 64, c16 = lane % 16, c0 = (blockIdx.y * W + threadIdx.x / 64) * 16, col = c0 + c16;
  long b, e;
  span(a, s, b, e);
  const long first = first_block(a, s), all = first_block(a, s + 1);
  if (e > b + (all - first) * B) e = b + (all - first) * B;
  State<KT> S;   // the gradient of the state behind a chunk
  S.load(a, a.dlast ? a.dlast + state_at(a, s, h) : nullptr, col);
  const T* D = (const T*)a.dout + (size_t)h * a.dv + col;
  const int chunks = (int)((e - b + C - 1) / C);
  const auto rows_in = [&](int c) { return e - b - (long)c * C < C ? (int)(e - b - (long)c * C) : C; };
  Ck next;
  Rows8<T> dnext;
  const auto fetch = [&](int c) {
    const long row = b + (long)c * C;
    next.fetch(a, row, rows_in(c), (size_t)(first + c / 2), c % 2, h, hk);
    dnext.fetch(D + row * a.dout_stride, a.dout_stride, rows_in(c), col < a.dv);
  };
  if (chunks > 0) {
    fetch(chunks - 1);
    next.put(sh[(chunks - 1) & 1]);
  }
  Rows8<T> d = dnext;
  __syncthreads();
  for (int c = chunks - 1; c >= 0; --c) {
    const typename Ck::Shared& t = sh[c & 1];
    const long row = b + (long)c * C;
    const int count = rows_in(c);
    if (c > 0) fetch(c - 1);
    if (c0 < a.dv) {
      if (c % 2 || c == chunks - 1) S.store(a, a.behind + state_at(a, (size_t)(first + c / 2), h), col);
      v4f ks[2] = {};
#pragma unroll
      for (int f = 0; f < KT; ++f) {
        const Frag<3> op = S.operand(f);
#pragma unroll
        for (int r = 0; r < 2; ++r) ks[r] = mma<3>(t.k.along_row(16 * r + c16, f), op, ks[r]);
      }
      float x[8], y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = widen(d.v[k]);
      const Frag<P> dop = split8<P>(x);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        ks[k / 4][k % 4] *= t.rest[chunk_row(k)];
        y[k] = a.scale * t.grow[chunk_row(k)] * x[k];
      }
      const Frag<3> od = split8<3>(y);
#pragma unroll
      for (int r = 0; r < 2; ++r) ks[r] = mma<3>(t.p.down(r, 0), dop, ks[r]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = ks[k / 4][k % 4];
        y[k] = t.beta[chunk_row(k)] * x[k];
      }
      const Frag<3> z = split8<3>(y);
      v4f nz[2] = {};
#pragma unroll
      for (int r = 0; r < 2; ++r) nz[r] = mma<3>(t.n.down(r, 0), z, nz[r]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] -= nz[k / 4][k % 4];
        if (col < a.dv && chunk_row(k) < count) a.x[(row + chunk_row(k)) * ((size_t)a.heads * a.dv) + (size_t)h * a.dv + col] = x[k];
        y[k] = -t.grow[chunk_row(k)] * t.beta[chunk_row(k)] * x[k];
      }
      const Frag<3> kd = split8<3>(y);
      const float whole = t.whole;
#pragma unroll
      for (int m = 0; m < 2 * KT; ++m) S.t[m] = mma<3>(t.k.down(m, 0), kd, mma<3>(t.q.down(m, 0), od, S.t[m] * whole));
    }
    if (c > 0) {
      next.put(sh[(c - 1) & 1]);
      d = dnext;
    }
    __syncthreads();
  }
  if (a.dh0) S.store(a, a.dh0 + state_at(a, s, h), col);
}

// ------------------------------------------------------------------ the gradients of a block
// Eight waves, each with 16 columns of dq and dk; the heads that share a key one behind the other.
template <class T, int KT>
__global__ __launch_bounds__(512) void delta_gradient_kernel(DeltaArgs a) {
  constexpr int P = In<T>::P, LD = KT * 32 + 8, LV = 32 + 8, LB = B + 8;
  struct Step {   // 32 columns of the values
    alignas(16) bf16 d[P][B][LV], y[3][B][LV], w[3][B][LV];
  };
  struct Pair {
    alignas(16) bf16 p[3][B][LB], m[3][B][LB];
  };
  __shared__ union {
    Step s;
    Pair m;
  } u;
  __shared__ Matrix<P, B, LD> kq;
  __shared__ double g[B];
  __shared__ float grow[B], rest[B], beta[B], dots[8][B], ends[8];
  Block w;
  const int hk = blockIdx.x % a.key_heads, group = a.heads / a.key_heads;
  if (!find_block(a, blockIdx.x / a.key_heads, w)) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c16 = lane % 16, q = lane / 16;
  const bool owner = wave < 2 * KT;
  const int kc = 16 * wave + c16;   // the column of dq and dk
  const T* K = row_of((const T*)a.k, w.row, a.k_stride) + (size_t)hk * a.dk;
  const T* Q = row_of((const T*)a.q, w.row, a.q_stride) + (size_t)hk * a.dk;
  const auto load_kq = [&](const T* p, size_t stride) {
#pragma unroll
    for (int j = 0; j < B * KT * 8 / 512; ++j) {
      const int i = threadIdx.x + j * 512, row = i / (KT * 8), four = i % (KT * 8);
      const long n = row < w.count ? a.dk - four * 4 : 0;
      v2u x[P];
      parts4(load_group<4>(p + (n > 0 ? row * stride + four * 4 : 0), n), x);
      kq.put(row, four, x);
    }
  };
  // operands in LDS whose columns lie in their order
  const auto along = [&](const auto& m, int row) {   // contracted over a step's 32 columns, eight of them in a row
    constexpr int PP = sizeof(m) / sizeof(m[0]);
    Frag<PP> r;
#pragma unroll
    for (int i = 0; i < PP; ++i) r.p[i] = *(const v4u*)&m[i][row][8 * q];
    return r;
  };
  const auto over_rows = [&](const bf16 (&m)[3][B][LB], int row, int f) {   // as `down` has its rows
    Frag<3> r;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const v2u lo = *(const v2u*)&m[i][row][32 * f + 4 * q], hi = *(const v2u*)&m[i][row][32 * f + 16 + 4 * q];
      r.p[i] = (v4u){lo.x, lo.y, hi.x, hi.y};
    }
    return r;
  };
  const auto turned = [&](const bf16 (&m)[3][B][LB], int tile, int f) {
    Frag<3> r;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const bf16* p = &m[i][32 * f + 4 * q + c16 / 4][16 * tile + 4 * (lane % 4)];
      const v2u lo = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p));
      const v2u hi = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 16 * LB)));
      r.p[i] = (v4u){lo.x, lo.y, hi.x, hi.y};
    }
    return r;
  };
  v4f sum_q[4] = {}, sum_k[4] = {};
  for (int h = hk * group; h < (hk + 1) * group; ++h) {
    __syncthreads();   // the head in front is done with LDS
    if (threadIdx.x < B) {
      const double* sums = sums_of(a, w.index, h);
      const double half = sums[C - 1], end = half + sums[B - 1], mine = sums[threadIdx.x] + (threadIdx.x >= C ? half : 0.0);
      g[threadIdx.x] = mine;
      grow[threadIdx.x] = expf((float)mine);
      rest[threadIdx.x] = expf((float)(end - mine));
      beta[threadIdx.x] = (int)threadIdx.x < w.count ? a.beta[(w.row + threadIdx.x) * a.beta_stride + h] : 0.f;
    }
    __syncthreads();
    const float* before = a.carry_in + a.carry_states + state_at(a, w.index, h);
    const float* behind = a.behind + state_at(a, w.index, h);
    const size_t wide = (size_t)a.heads * a.dv;
    v4f dq[4] = {}, dr[4] = {}, dc[4] = {};   // by the rows' own decays: q's, k's where it reads the state, k's where it writes it
    v4f pair[3] = {};                         // tiles of dO W^T (0 .. 9) and Y W^T (10 .. 19) on and below the diagonal
    float ss = 0.f, dbeta = 0.f;
    const int row = threadIdx.x / 8;
    const bool in = row < w.count;
    for (int v0 = 0; v0 < a.dv; v0 += 32) {
      const long n = in ? a.dv - v0 - 4 * (int)(threadIdx.x % 8) : 0;
      const size_t at = n > 0 ? (size_t)h * a.dv + v0 + 4 * (threadIdx.x % 8) : 0;
      const size_t r = in ? w.row + row : w.row;
      const Vec<T, 4> d = load_group<4>((const T*)a.dout + r * a.dout_stride + at, n);
      const Vec<float, 4> ev = load_group<4>(a.carry_in + r * wide + at, n), xv = load_group<4>(a.x + r * wide + at, n);
      float s0[8] = {}, s1[8] = {};
      if (kc < a.dk && owner) {
        const long left = a.dv - v0 - 8 * q;
#pragma unroll
        for (int k = 0; k < 8; k += 4) {
          const size_t o = left > k ? (size_t)kc * a.dv + v0 + 8 * q + k : 0;
          const Vec<float, 4> x = load_group<4>(before + o, left - k), y = load_group<4>(behind + o, left - k);
#pragma unroll
          for (int i = 0; i < 4; ++i) s0[k + i] = get(x, i), s1[k + i] = get(y, i);
        }
      }
      float y[4], e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dbeta = fmaf(get(xv, i), get(ev, i), dbeta);
        y[i] = beta[row] * get(xv, i);
        e[i] = beta[row] * get(ev, i);
      }
      if (n > 0) store_vec((T*)a.dvalue + r * a.dv_stride + at, pack<T>(y), n);
      v2u x[3], z[P];
      parts4(d, z);
#pragma unroll
      for (int i = 0; i < P; ++i) *(v2u*)&u.s.d[i][row][4 * (threadIdx.x % 8)] = z[i];
      split4<3>(y, x);
#pragma unroll
      for (int i = 0; i < 3; ++i) *(v2u*)&u.s.y[i][row][4 * (threadIdx.x % 8)] = x[i];
      split4<3>(e, x);
#pragma unroll
      for (int i = 0; i < 3; ++i) *(v2u*)&u.s.w[i][row][4 * (threadIdx.x % 8)] = x[i];
      __syncthreads();
      if (owner) {
        const Frag<3> f0 = split8<3>(s0), f1 = split8<3>(s1);
#pragma unroll
        for (int k = 0; k < 8; ++k) ss = fmaf(s0[k], s1[k], ss);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          dq[t] = mma<3>(along(u.s.d, 16 * t + c16), f0, dq[t]);
          dr[t] = mma<3>(along(u.s.y, 16 * t + c16), f0, dr[t]);
          dc[t] = mma<3>(along(u.s.w, 16 * t + c16), f1, dc[t]);
        }
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int t = wave + 8 * k, o = t % 10, it = o >= 6 ? 3 : o >= 3 ? 2 : o >= 1 ? 1 : 0, jt = o - it * (it + 1) / 2;
        if (t < 10) pair[k] = mma<3>(along(u.s.d, 16 * it + c16), along(u.s.w, 16 * jt + c16), pair[k]);
        else if (t < 20) pair[k] = mma<3>(along(u.s.y, 16 * it + c16), along(u.s.w, 16 * jt + c16), pair[k]);
      }
      __syncthreads();
    }
    // dbeta: the eight threads of a row
    dbeta = group_sum<8>(dbeta);
    if (in && threadIdx.x % 8 == 0) a.dbeta[(w.row + row) * a.dbeta_stride + h] = dbeta;
    // the pairs' gradients into LDS, and zeros above the diagonal where an operand has them
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int t = wave + 8 * k, o = t % 10, it = o >= 6 ? 3 : o >= 3 ? 2 : o >= 1 ? 1 : 0, jt = o - it * (it + 1) / 2;
      if (t >= 24) continue;
      const int zero = t - 20;   // 20 .. 23: the tiles (0, 1) and (2, 3) of both
      const int i0 = 16 * (zero >= 0 ? zero / 2 * 2 : it), j = 16 * (zero >= 0 ? zero / 2 * 2 + 1 : jt) + c16;
      bf16(*m)[B][LB] = (zero >= 0 ? zero % 2 : t >= 10) ? u.m.m : u.m.p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i0 + 4 * q + i;
        float x = 0.f;
        if (zero < 0 && t < 10 && r >= j) x = a.scale * expf((float)(g[r] - g[j])) * pair[k][i];
        if (zero < 0 && t >= 10 && r > j) x = -expf((float)(g[r] - g[j])) * pair[k][i];
        unsigned p[3];
        split2<3>(x, 0.f, p);
#pragma unroll
        for (int z = 0; z < 3; ++z) *(unsigned short*)&m[z][r][j] = (unsigned short)p[z];
      }
    }
    float tail = 0.f;   // what the sum of all decays of the block is owed
    v4f kv[4], qv[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * t + 4 * q + i;
        const bool there = owner && kc < a.dk && r < w.count;
        kv[t][i] = there ? widen(K[r * a.k_stride + kc]) : 0.f;
        qv[t][i] = there ? widen(Q[r * a.q_stride + kc]) : 0.f;
        dq[t][i] *= a.scale * grow[r];
        dr[t][i] *= -grow[r];
        dc[t][i] *= rest[r];
        tail = fmaf(kv[t][i], dc[t][i], tail);
      }
    tail = group_sum<64>(fmaf(expf((float)g[B - 1]), ss, tail));
    if (lane == 0) ends[wave] = tail;
    load_kq(Q, a.q_stride);
    __syncthreads();
    if (owner)
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Frag<P> b = kq.down(wave, 32 * f);
#pragma unroll
        for (int t = 0; t < 2 * f + 2; ++t) dc[t] = mma<3>(turned(u.m.p, t, f), b, dc[t]);
      }
    __syncthreads();
    load_kq(K, a.k_stride);
    __syncthreads();
    if (owner) {
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Frag<P> b = kq.down(wave, 32 * f);
#pragma unroll
        for (int t = 0; t < 2 * f + 2; ++t) dc[t] = mma<3>(turned(u.m.m, t, f), b, dc[t]);
#pragma unroll
        for (int t = 2 * f; t < 4; ++t) {
          dq[t] = mma<3>(over_rows(u.m.p, 16 * t + c16, f), b, dq[t]);
          dr[t] = mma<3>(over_rows(u.m.m, 16 * t + c16, f), b, dr[t]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = group_sum<16>(qv[t][i] * dq[t][i] + kv[t][i] * (dr[t][i] - dc[t][i]));
        if (c16 == 0) dots[wave][16 * t + 4 * q + i] = x;
        sum_q[t][i] += dq[t][i];
        sum_k[t][i] += dr[t][i] + dc[t][i];
      }
    __syncthreads();
    if (wave == 0) {
      float x = 0.f, end = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) x += dots[i][lane], end += ends[i];
      if (lane == B - 1) x += end;
#pragma unroll
      for (int d = 1; d < B; d *= 2) {
        const float down = __shfl_down(x, d, 64);
        if (lane + d < B) x += down;
      }
      if (lane < w.count) a.ddecay[(w.row + lane) * a.ddecay_stride + h] = x;
    }
  }
  if (owner && kc < a.dk)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * t + 4 * q + i;
        if (r >= w.count) continue;
        ((T*)a.dq)[(w.row + r) * a.dq_stride + (size_t)hk * a.dk + kc] = (T)sum_q[t][i];
        ((T*)a.dkey)[(w.row + r) * a.dk_stride + (size_t)hk * a.dk + kc] = (T)sum_k[t][i];
      }
}

// ------------------------------------------------------------------ one row of every sequence
// The state once through registers: 32 columns to a workgroup, four to a thread, rows 32 apart; k^T S and q^T S are formed together, and with
// S' = a S + beta k e^T, q^T S' = a q^T S + beta (q.k) e needs no second pass.
template <class T>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaStepArgs a) {
  constexpr int NR = DELTA_MAX_KEY / 32;
  __shared__ float part[4][8][8];   // wave, column group, k^T S and q^T S
  __shared__ float dot[4];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads), x = threadIdx.x % 8, y = threadIdx.x / 8, lane = threadIdx.x % 64;
  const size_t row = blockIdx.x / a.heads;
  const int col = blockIdx.y * 32 + 4 * x;
  const long n = a.dv - col;
  float* S = a.state + row * a.state_stride + (size_t)h * a.dk * a.dv;
  Vec<float, 4> s[NR];
  float k[NR], q[NR];
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const int r = y + 32 * j;
    const bool in = r < a.dk;
    s[j] = load_group<4>(S + (in && n > 0 ? (size_t)r * a.dv + col : 0), in ? n : 0);
    k[j] = in ? widen(row_of((const T*)a.k, row, a.k_stride)[(size_t)hk * a.dk + r]) : 0.f;
    q[j] = in ? widen(row_of((const T*)a.q, row, a.q_stride)[(size_t)hk * a.dk + r]) : 0.f;
  }
  const Vec<T, 4> v = load_group<4>(row_of((const T*)a.v, row, a.v_stride) + (size_t)h * a.dv + (n > 0 ? col : 0), n);
  const float keep = expf(a.decay[row * a.decay_stride + h]), beta = a.beta[row * a.beta_stride + h];
  float sum[8] = {}, qk = 0.f;
#pragma unroll
  for (int j = 0; j < NR; ++j) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[i] = fmaf(k[j], get(s[j], i), sum[i]);
      sum[4 + i] = fmaf(q[j], get(s[j], i), sum[4 + i]);
    }
    qk = fmaf(q[j], k[j], qk);
  }
#pragma unroll
  for (int d = 8; d < 64; d *= 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] += __shfl_xor(sum[i], d, 64);
    qk += __shfl_xor(qk, d, 64);
  }
  if (lane < 8)
#pragma unroll
    for (int i = 0; i < 8; ++i) part[threadIdx.x / 64][x][i] = sum[i];
  if (lane == 0) dot[threadIdx.x / 64] = qk;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = (part[0][x][i] + part[1][x][i]) + (part[2][x][i] + part[3][x][i]);
  qk = (dot[0] + dot[1]) + (dot[2] + dot[3]);
  float e[4], o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e[i] = beta * (get(v, i) - keep * sum[i]);
    o[i] = a.scale * fmaf(qk, e[i], keep * sum[4 + i]);
  }
  if (n <= 0) return;
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    const int r = y + 32 * j;
    if (r >= a.dk) continue;
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = fmaf(k[j], e[i], keep * get(s[j], i));
    store_vec(S + (size_t)r * a.dv + col, pack<float>(z), n);
  }
  if (y == 0 && a.o) store_vec(row_of((T*)a.o, row, a.o_stride) + (size_t)h * a.dv + col, pack<T>(o), n);
}

// ------------------------------------------------------------------ launches
struct Sizes {
  size_t blocks, first, matrices, sums, x, behind, bytes;   // offsets into the workspace
};
Sizes sizes_of(size_t rows, size_t n, size_t heads, size_t dk, size_t dv, bool backward) {
  Sizes s;
  s.blocks = rows / B + (n < rows ? n : rows);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t p = at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  s.first = take((n + 1) * sizeof(int));
  s.matrices = take(s.blocks * heads * 4 * C * C * sizeof(float));
  s.sums = take(s.blocks * heads * B * sizeof(double));
  s.x = take(backward ? rows * heads * dv * sizeof(float) : 0);
  s.behind = take(backward ? s.blocks * heads * dk * dv * sizeof(float) : 0);
  s.bytes = at;
  return s;
}

void lay_out(DeltaArgs& a, bool backward) {
  const Sizes s = sizes_of(a.rows, a.n_seq, a.heads, a.dk, a.dv, backward);
  char* w = (char*)a.workspace;
  a.blocks = s.blocks;
  a.first = (int*)(w + s.first);
  a.matrices = (float*)(w + s.matrices);
  a.sums = (double*)(w + s.sums);
  a.x = (float*)(w + s.x);
  a.behind = (float*)(w + s.behind);
  a.carry_states = a.rows * a.heads * a.dv;
}

hipError_t plan(const DeltaArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.begin) e = launch(delta_plan_kernel, dim3(1), dim3(PLAN), 0, stream, a);
  const size_t groups = (a.rows + 3) / 4;
  if (e == hipSuccess && a.zero_others && a.rows && (a.begin || !a.n_seq))
    e = launch(delta_zero_kernel, dim3((unsigned)(groups < 65536 ? groups : 65536)), dim3(256), 0, stream, a);
  return e;
}

template <class T, int KT>
hipError_t prepare(const DeltaArgs& a, hipStream_t stream) {
  return launch(delta_prepare_kernel<T, KT>, dim3((unsigned)(a.blocks * a.heads)), dim3(256), 0, stream, a);
}

template <class T, int KT>
hipError_t forward(const DeltaArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.blocks) e = prepare<T, KT>(a, stream);
  if (e != hipSuccess || !a.n_seq) return e;
  const unsigned x = (unsigned)(a.n_seq * a.heads), tiles = (a.dv + 15) / 16;
  if (tiles <= 4) return launch(delta_forward_kernel<T, KT, 4>, dim3(x, 1), dim3(256), 0, stream, a);
  return launch(delta_forward_kernel<T, KT, 8>, dim3(x, (tiles + 7) / 8), dim3(512), 0, stream, a);
}

template <class T, int KT>
hipError_t backward(const DeltaArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.blocks) e = prepare<T, KT>(a, stream);
  if (e != hipSuccess || !a.n_seq) return e;
  const unsigned x = (unsigned)(a.n_seq * a.heads), tiles = (a.dv + 15) / 16;
  if (tiles <= 4) e = launch(delta_backward_kernel<T, KT, 4>, dim3(x, 1), dim3(256), 0, stream, a);
  else e = launch(delta_backward_kernel<T, KT, 8>, dim3(x, (tiles + 7) / 8), dim3(512), 0, stream, a);
  if (e != hipSuccess || !a.blocks) return e;
  return launch(delta_gradient_kernel<T, KT>, dim3((unsigned)(a.blocks * a.key_heads)), dim3(512), 0, stream, a);
}

#define BY_KEY(CALL)                  \
  if (a.dk <= 32) return CALL(1);     \
  if (a.dk <= 64) return CALL(2);     \
  return CALL(4);

}  // namespace

extern "C" size_t amp_delta_blocks(size_t rows, size_t n) { return sizes_of(rows, n, 1, 1, 1, false).blocks; }
extern "C" size_t amp_delta_workspace_bytes(size_t rows, size_t n, size_t heads, size_t dk, size_t dv, int backward) {
  return sizes_of(rows, n, heads, dk, dv, backward).bytes;
}

extern "C" hipError_t amp_delta_forward_launch(int dtype, const DeltaArgs* args, hipStream_t stream) {
  DeltaArgs a = *args;
  lay_out(a, false);
  const hipError_t e = plan(a, stream);
  if (e != hipSuccess) return e;
#define DELTA_F(KT) forward<T, KT>(a, stream)
  OPS_BY_TYPE(dtype, BY_KEY(DELTA_F));
}

extern "C" hipError_t amp_delta_backward_launch(int dtype, const DeltaArgs* args, hipStream_t stream) {
  DeltaArgs a = *args;
  lay_out(a, true);
  const hipError_t e = plan(a, stream);
  if (e != hipSuccess) return e;
#define DELTA_B(KT) backward<T, KT>(a, stream)
  OPS_BY_TYPE(dtype, BY_KEY(DELTA_B));
}

extern "C" hipError_t amp_delta_step_launch(int dtype, const DeltaStepArgs* a, hipStream_t stream) {
  const dim3 grid((unsigned)(a->rows * a->heads), (unsigned)((a->dv + 31) / 32));
  OPS_BY_TYPE(dtype, return launch(delta_step_kernel<T>, grid, dim3(256), 0, stream, *a));
}
