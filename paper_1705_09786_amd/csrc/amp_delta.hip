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
// Kernels: the plan, the blocks of 64 rows in front of every sequence; per block and head, N and P of its two chunks; where sequences are
// long, the maps of their segments and the chain over those; the chain over the chunks, a workgroup for each sequence (or segment) and
// head, whose waves have 16 columns of the state each in registers all along: a state is both result and operand of the matrix instructions
// in the layout that it has there, so that nothing but K, Q, N and P passes through LDS; backward, the chain the other way; and per
// block, the gradients.
//
// Products run on the bf16 matrix instructions, whose operands hold 8 bits: a number is the sum of up to three of them (24 bits, as in 32-bit
// arithmetic; an input in bf16 is one, in fp16 two), and of a product's partial products those are taken that reach 2^-24 of it. That is
// three instructions for an input in bf16 with a state, six for a state with a state, each of 16 times the rate of the 32-bit ones.
//
// What bounds it: not HBM. A chunk of the chain takes 4 us on a compute unit (16,384 rows in 24 sequences, 16 heads of 128 x 128 bf16: 235 us
// either way): vector instructions (a state's parts are formed anew for every chunk) keep the SIMDs busy for 45 % of that, the
// matrix instructions for 30 %, and what is left is the two of them waiting for one another and for LDS, with two waves to a SIMD for want of
// registers. The gradients (430 us of that case) wait for memory with one workgroup to a compute unit.
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

// N pairs of numbers in parts: u[part][pair].
template <int P, int N>
__device__ __forceinline__ void split(float (&a)[N], float (&b)[N], unsigned (&u)[P][N]) {
  // what a part leaves of its number, exactly, in one instruction: a - 1 u.lo - 0 u.hi. (The factors pass through registers: as a
  // constant -1 the instruction would take the upper half.) Part by part over all pairs: its result is late for the next instruction.
  unsigned lo = 0xbf80u, hi = 0xbf800000u;
  asm("" : "+s"(lo));
  asm("" : "+s"(hi));
#pragma unroll
  for (int i = 0; i < P; ++i) {
#pragma unroll
    for (int k = 0; k < N; ++k) u[i][k] = pack2(a[k], b[k], bf16());
    if (i + 1 < P)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        a[k] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, u[i][k]), __builtin_bit_cast(v2bf, lo), a[k], false);
        b[k] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, u[i][k]), __builtin_bit_cast(v2bf, hi), b[k], false);
      }
  }
}
template <int P>
__device__ __forceinline__ Frag<P> split8(const float (&x)[8]) {
  float a[4] = {x[0], x[2], x[4], x[6]}, b[4] = {x[1], x[3], x[5], x[7]};
  unsigned u[P][4];
  split<P, 4>(a, b, u);
  Frag<P> f;
#pragma unroll
  for (int i = 0; i < P; ++i) f.p[i] = (v4u){u[i][0], u[i][1], u[i][2], u[i][3]};
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

// The same for two operands a side by side, whose results wait for nothing of one another.
template <int ORDER, int PA, int PB>
__device__ __forceinline__ void mma2(const Frag<PA> (&a)[2], const Frag<PB>& b, v4f (&c)[2]) {
#pragma unroll
  for (int s = ORDER - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i)
      if (s - i >= 0 && s - i < PB)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          c[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a[r].p[i]), __builtin_bit_cast(v8bf, b.p[s - i]), c[r], 0, 0, 0);
}

// The sum over a lane's 16 (8), by rotations within them: lane 0's is added up in the same order always.
template <int W>
__device__ __forceinline__ float rotate(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x120 + W, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float v) {
  v += rotate<8>(v);
  v += rotate<4>(v);
  v += rotate<2>(v);
  return v + rotate<1>(v);
}

// Matrices in LDS. An operand is read along its rows, 8 bytes from each of 16 rows at a time, or down its columns, transposed, 32 bytes from each of
// four rows: rows 8 words more than a multiple of 32 apart, and 2 between fours of them, put either's 16 lanes on 32 banks of their own.
template <int P, int ROWS, int COLS>
struct Matrix {
  static constexpr int LD = COLS + 16;
  alignas(16) bf16 at[P][ROWS * LD + 16];
  static __device__ __forceinline__ int place(int row, int col) { return row * LD + row / 4 % 4 * 4 + col; }
  // the operand whose lane has row row0 + lane % 16, contracted over the columns 32 f ..: 4 q .. and 16 + 4 q ..
  __device__ __forceinline__ Frag<P> along(int row0, int f) const {
    const int o = place(row0 + threadIdx.x % 16, 32 * f + threadIdx.x % 64 / 16 * 4);
    Frag<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const v2u lo = *(const v2u*)&at[i][o], hi = *(const v2u*)&at[i][o + 16];
      r.p[i] = (v4u){lo.x, lo.y, hi.x, hi.y};
    }
    return r;
  }
  // the operand whose lane has column 16 tile + lane % 16, contracted over the rows row0 ..: four rows of 16 columns to 16 lanes
  __device__ __forceinline__ Frag<P> down(int tile, int row0) const {
    const int lane = threadIdx.x % 64, row = row0 + lane / 16 * 4 + lane % 16 / 4, col = 16 * tile + 4 * (lane % 4);
    Frag<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const v2u lo = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)&at[i][place(row, col)]));
      const v2u hi = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)&at[i][place(row + 16, col)]));
      r.p[i] = (v4u){lo.x, lo.y, hi.x, hi.y};
    }
    return r;
  }
  // four columns from 4 `four` on
  __device__ __forceinline__ void put(int row, int four, const v2u (&u)[P]) {
#pragma unroll
    for (int i = 0; i < P; ++i) *(v2u*)&at[i][place(row, 4 * four)] = u[i];
  }
};

// Nothing moves across: the reads in front are on their way while what follows is worked on. (Not where four waves share a SIMD: they have
// half the registers, and one another to wait with.)
template <bool PIN>
__device__ __forceinline__ void on_their_way() {
  if constexpr (PIN) __builtin_amdgcn_sched_barrier(0);
}

template <int P>
__device__ __forceinline__ void split4(const float (&x)[4], v2u (&u)[P]) {
  float a[2] = {x[0], x[2]}, b[2] = {x[1], x[3]};
  unsigned w[P][2];
  split<P, 2>(a, b, w);
#pragma unroll
  for (int i = 0; i < P; ++i) u[i] = (v2u){w[i][0], w[i][1]};
}
__device__ __forceinline__ void parts4(const Vec<bf16, 4>& v, v2u (&u)[1]) { u[0] = v.u; }
template <class T, int P>
__device__ __forceinline__ void parts4(const Vec<T, 4>& v, v2u (&u)[P]) {
  const float x[4] = {get(v, 0), get(v, 1), get(v, 2), get(v, 3)};
  split4<P>(x, u);
}

// base + bytes, for a base that is the same for all lanes.
template <class T>
__device__ __forceinline__ const T* past(const T* base, unsigned bytes) { return (const T*)((const char*)base + bytes); }
template <class T>
__device__ __forceinline__ T* past(T* base, unsigned bytes) { return (T*)((char*)base + bytes); }

// Four elements, n and later replaced by zeros; p can be read where n is 0 as well. By `fours`, the same for all lanes: FOURS, n is a multiple of 4, as
// where dk and dv are; ROWS, of a row's last elements at least four are there: they are read and moved down; NARROW, one by one. (A
// branch for every count of elements costs the kernels' loops registers, which they spill.)
enum { NARROW = 0, ROWS = 1, FOURS = 2 };
template <class T>
__device__ __forceinline__ Vec<T, 4> load_four(const T* p, int n, int fours) {
  Vec<T, 4> v;
  v.u = (typename Vec<T, 4>::U)0u;
  if (fours == FOURS) {
    if (n > 0) v.u = *(const typename Vec<T, 4>::Any*)p;
  } else if (fours == ROWS) {
    const int gone = n <= 0 || n >= 4 ? 0 : 4 - n;
    if (n > 0) v.u = *(const typename Vec<T, 4>::Any*)(p - gone);
    if constexpr (sizeof(T) == 2) {
      const unsigned long x = ((unsigned long)v.u[1] << 32 | v.u[0]) >> (16 * gone);
      v.u[0] = (unsigned)x, v.u[1] = (unsigned)(x >> 32);
    } else {
      if (gone & 1) v.u = (v4u){v.u[1], v.u[2], v.u[3], 0u};
      if (gone & 2) v.u = (v4u){v.u[2], v.u[3], 0u, 0u};
    }
  } else {
    unsigned e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const T* at = p + (k < n ? k : 0);
      const unsigned x = sizeof(T) == 2 ? (unsigned)*(const unsigned short*)at : *(const unsigned*)at;
      e[k] = k < n ? x : 0u;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (sizeof(T) == 2) v.u[k / 2] |= e[k] << (16 * (k & 1));
      else v.u[k] = e[k];
  }
  return v;
}
template <class T>
__device__ __forceinline__ void store_four(T* p, Vec<T, 4> v, int n, int fours) {
  if (fours == FOURS) {
    if (n > 0) *(typename Vec<T, 4>::Any*)p = v.u;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) {
        if (sizeof(T) == 2) ((unsigned short*)p)[k] = (unsigned short)(v.u[k / 2] >> (16 * (k & 1)));
        else ((unsigned*)p)[k] = v.u[k];
      }
  }
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
__host__ __device__ inline long blocks_of(long rows) { return (rows + B - 1) / B; }
// Blocks in front of a sequence, at most the workspace's number of them. (That number, a.blocks, is a bound: one sequence of a multiple of 64 rows
// has one block less.)
__device__ __forceinline__ long first_block(const DeltaArgs& a, size_t s) { return a.begin ? a.first[s] : s ? blocks_of((long)a.rows) : 0; }

// `first`: the plan's or, without sequences' bounds, nothing.
__device__ __forceinline__ bool search_block(const DeltaArgs& a, const int* first, size_t index, Block& w) {
  const auto at = [&](size_t s) { return first ? (long)first[s] : first_block(a, s); };
  size_t lo = 0, hi = a.n_seq;   // first[lo] <= index < first[hi]
  if ((long)index >= at(hi)) return false;
  while (hi - lo > 1) {
    const size_t mid = (lo + hi) / 2;
    (at(mid) <= (long)index ? lo : hi) = mid;
  }
  long b, e;
  span(a, lo, b, e);
  w.row = b + ((long)index - at(lo)) * B;
  w.count = e - w.row < B ? (int)(e - w.row) : B;
  w.index = index;
  return w.count > 0;
}

// The same from the plan's table: a block's first row and its rows, 0 where there is none.
__device__ __forceinline__ bool find_block(const DeltaArgs& a, size_t index, Block& w) {
  if (!a.begin) return search_block(a, nullptr, index, w);
  w.row = a.table[2 * index], w.count = a.table[2 * index + 1], w.index = index;
  return w.count > 0;
}

// N and P of a chunk; e^G, e^{G_end - G} and beta of a block's rows and e^{G_end} of its two chunks; the sums G of decays (in 64 bits:
// differences of far sums decide about near rows).
__device__ __forceinline__ float* matrices_of(const DeltaArgs& a, size_t block, int h, int chunk) {
  return a.matrices + ((block * a.heads + h) * 2 + chunk) * (2 * C * C);
}
__device__ __forceinline__ float* scalars_of(const DeltaArgs& a, size_t block, int h) { return a.scalars + (block * a.heads + h) * (4 * B); }
__device__ __forceinline__ double* sums_of(const DeltaArgs& a, size_t block, int h) { return a.sums + (block * a.heads + h) * B; }
// What the gradients are formed from lies block by block and head by head in tiles of 16 columns, as the chain's waves have them, so that both
// sides read and write memory in one piece: E and X 64 rows to a tile, states dk; columns behind the last are zeros.
__device__ __forceinline__ int tiled_columns(const DeltaArgs& a) { return (a.dv + 15) / 16 * 16; }
__device__ __forceinline__ size_t rows_at(const DeltaArgs& a, size_t block, int h) { return (block * a.heads + h) * ((size_t)B * tiled_columns(a)); }
__device__ __forceinline__ size_t tiles_at(const DeltaArgs& a, size_t block, int h) { return (block * a.heads + h) * ((size_t)a.dk * tiled_columns(a)); }

__device__ __forceinline__ size_t state_at(const DeltaArgs& a, size_t index, int h) { return (index * a.heads + h) * ((size_t)a.dk * a.dv); }

// ------------------------------------------------------------------ plan
// A long sequence is cut into segments whose chains run side by side, where that is sooner: every segment but its last passes once more
// without outputs, for the map from the state in front of it to the one behind it (dk columns beside the dv), and a short chain over the
// segments joins those. `longest` and `all` blocks, `work` workgroups to a block's chain: the chain alone takes the longest sequence's blocks,
// or all of them over the compute units; with segments two and a half times the latter and some blocks' time for the join. Blocks of
// a segment; 1 << 30: whole sequences.
__host__ __device__ inline long segment_blocks(long longest, long all, long work) {
  const long share = (all * work + 255) / 256;
  if (longest < 24 || longest <= share * 5 / 2 + 8) return (long)1 << 30;
  long root = DELTA_SEGMENT;   // a segment's blocks pass twice, and are a step of the join
  while (root * root * 4 < longest) ++root;
  return root > share ? root : share;
}
// Segments of a sequence, the whole of one that is not cut.
__host__ __device__ inline long segments_of(long blocks, long size) { return blocks > size ? (blocks + size - 1) / size : 1; }

struct Job {
  size_t s;          // its sequence
  long from, to;     // its blocks, counted in the sequence
  bool first, last;  // of the sequence's segments
  size_t slot;       // of a sequence that is cut: where its map and the state in front of it are
};
__device__ __forceinline__ size_t first_slot(const DeltaArgs& a, size_t s) { return a.begin ? a.first_slot[s] : 0; }
__device__ __forceinline__ bool whole_sequences(const DeltaArgs& a) { return a.begin && a.first_segment[a.n_seq] == (int)a.n_seq; }
// Segment `index` of all of them.
__device__ __forceinline__ bool find_job(const DeltaArgs& a, size_t index, Job& w) {
  if (!a.segments || whole_sequences(a)) {   // no sequence is cut: nothing to search for
    if (index >= a.n_seq) return false;
    if (a.begin && a.n_seq <= DELTA_ORDER) index = a.order[index];
    w.s = index, w.from = 0, w.to = first_block(a, index + 1) - first_block(a, index), w.first = w.last = true, w.slot = 0;
    return true;
  }
  size_t lo = 0, hi = a.n_seq;
  long size = a.segment;
  if (a.begin) {
    size = a.first_segment[a.n_seq + 1];
    if ((long)index >= a.first_segment[hi]) return false;
    while (hi - lo > 1) {
      const size_t mid = (lo + hi) / 2;
      (a.first_segment[mid] <= (long)index ? lo : hi) = mid;
    }
    index -= a.first_segment[lo];
  }
  const long blocks = first_block(a, lo + 1) - first_block(a, lo), count = segments_of(blocks, size);
  if ((long)index >= count) return false;
  w.s = lo, w.from = (long)index * size, w.to = w.from + size < blocks ? w.from + size : blocks;
  w.first = index == 0, w.last = (long)index + 1 == count;
  w.slot = count > 1 ? first_slot(a, lo) + index : 0;
  return true;
}

constexpr int PLAN = 1024, NEAR = 4096;
// Sums in front of every thread's value; `base` goes on by the sum of all.
__device__ __forceinline__ long sum_in_front(long mine, long& base, long (&part)[PLAN / 64]) {
  long sum = mine;
  for (int d = 1; d < 64; d *= 2) {
    const long up = __shfl_up(sum, d, 64);
    if ((int)(threadIdx.x & 63) >= d) sum += up;
  }
  if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  long front = base + sum - mine;
  for (int w = 0; w < PLAN / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) front += part[w];
    base += part[w];
  }
  __syncthreads();
  return front;
}

__global__ __launch_bounds__(PLAN) void delta_plan_kernel(DeltaArgs a, long work) {
  __shared__ long part[PLAN / 64];
  __shared__ int copy[NEAR + 1];   // of `first`, where it fits
  const int* near = a.n_seq <= NEAR ? copy : a.first;
  const long most = (long)a.blocks;
  long base = 0, longest = 0, inside = 0;
  for (size_t s0 = 0; s0 < a.n_seq; s0 += PLAN) {
    const size_t s = s0 + threadIdx.x;
    long b = 0, e = 0;
    if (s < a.n_seq) span(a, s, b, e);
    const long mine = blocks_of(e - b), at = sum_in_front(mine, base, part);
    longest = mine > longest ? mine : longest;
    inside += e - b;
    if (s < a.n_seq) {
      a.first[s] = (int)(at < most ? at : most);
      if (a.n_seq <= NEAR) copy[s] = a.first[s];
    }
  }
  const long all = base < most ? base : most;
  long sum = 0;
  sum_in_front(inside, sum, part);
  if (threadIdx.x == 0) {
    a.first[a.n_seq] = (int)all;
    if (a.n_seq <= NEAR) copy[a.n_seq] = (int)all;
    a.first[a.n_seq + 1] = sum == (long)a.rows;   // no rows of no sequence
  }
  __syncthreads();
  for (size_t i = threadIdx.x; i < a.blocks; i += PLAN) {
    Block w;
    const bool in = search_block(a, near, i, w);
    a.table[2 * i] = in ? (int)w.row : 0, a.table[2 * i + 1] = in ? w.count : 0;
  }
  if (a.n_seq <= DELTA_ORDER && threadIdx.x < a.n_seq) {   // the longest sequences first: 24 of up to 1,350 rows on 16 heads 230 us for 300
    const int mine = near[threadIdx.x + 1] - near[threadIdx.x];
    int front = 0;
    for (int s = 0; s < (int)a.n_seq; ++s) {
      const int other = near[s + 1] - near[s];
      front += other > mine || (other == mine && s < (int)threadIdx.x);
    }
    a.order[front] = (int)threadIdx.x;
  }
  if (!a.segments) return;
  for (int d = 1; d < 64; d *= 2) longest = max(longest, __shfl_xor(longest, d, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = longest;
  __syncthreads();
  for (int w = 0; w < PLAN / 64; ++w) longest = max(longest, part[w]);
  __syncthreads();
  // segments, and in the upper half those of sequences that are cut; of more of these than there are places, as only sequences out of order
  // have, none is cut
  for (long size = segment_blocks(longest < all ? longest : all, all, work);; size = (long)1 << 30) {
    base = 0;
    for (size_t s0 = 0; s0 < a.n_seq; s0 += PLAN) {
      const size_t s = s0 + threadIdx.x;
      long blocks = 0;
      if (s < a.n_seq) blocks = near[s + 1] - near[s];   // written by this workgroup, a barrier ago
      const long count = s < a.n_seq ? segments_of(blocks, size) : 0, at = sum_in_front(count > 1 ? count << 32 | count : count, base, part);
      if (s < a.n_seq) a.first_segment[s] = (int)at, a.first_slot[s] = (int)(at >> 32);
    }
    if (threadIdx.x == 0) a.first_segment[a.n_seq] = (int)base, a.first_segment[a.n_seq + 1] = (int)size;
    if (base >> 32 <= (long)a.slots) break;
  }
}

// Rows of no sequence: a wave to a row, zeros in every output.
__global__ __launch_bounds__(256) void delta_zero_kernel(DeltaArgs a) {
  if (a.n_seq && a.first[a.n_seq + 1]) return;
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
// 4,480 blocks and heads of 128 bf16 in 50 us: 3 TB/s of keys and queries read and matrices written.
// e^x of a difference of sums: half a step of its exponent and the instruction's own.
__device__ __forceinline__ float power(double x) { return __builtin_amdgcn_exp2f((float)(x * 1.4426950408889634)); }

// N = (1 + M beta)^-1 M of a chunk in halves of 16 rows: those on the diagonal row after row, N = M - (M beta) N, a lane to a column; the one
// below them from two products, N21 = W - N22 beta W with W = M21 - M21 beta N11.
template <class T, int KT>
__global__ __launch_bounds__(256) void delta_prepare_kernel(DeltaArgs a) {
  constexpr int P = In<T>::P, LM = C + 4;
  __shared__ union {
    struct {
      Matrix<P, B, KT * 32> k, q;
    } in;
    struct {
      alignas(16) float mat[2][2][C][LM];   // chunk; M beta (first K K^T), M (first Q K^T)
      float n[4][16][17];                   // the halves on the diagonal
    } m;
  } u;
  __shared__ double g[B];
  __shared__ float beta[B];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads);
  Block w;
  if (!find_block(a, blockIdx.x / a.heads, w)) return;
  const T* K = row_of((const T*)a.k, w.row, a.k_stride) + (size_t)hk * a.dk;
  const T* Q = row_of((const T*)a.q, w.row, a.q_stride) + (size_t)hk * a.dk;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  constexpr int PER = B * KT * 8 / 256;
  Vec<T, 4> kv[PER], qv[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int x = threadIdx.x + j * 256, row = x / (KT * 8), four = x % (KT * 8), n = row < w.count ? a.dk - four * 4 : 0;
    kv[j] = load_four(past(K, n > 0 ? (row * (unsigned)a.k_stride + four * 4) * (unsigned)sizeof(T) : 0u), n, a.fours);
    qv[j] = load_four(past(Q, n > 0 ? (row * (unsigned)a.q_stride + four * 4) * (unsigned)sizeof(T) : 0u), n, a.fours);
  }
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
    const double end = __shfl(sum, C - 1, C);
    float* f = scalars_of(a, w.index, h);
    f[lane] = power(sum);
    f[B + lane] = power(end - sum);
    f[2 * B + lane] = bt;
    if (lane % C == 0) f[3 * B + lane / C] = power(end);
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int x = threadIdx.x + j * 256;
    v2u y[P];
    parts4(kv[j], y);
    u.in.k.put(x / (KT * 8), x % (KT * 8), y);
    parts4(qv[j], y);
    u.in.q.put(x / (KT * 8), x % (KT * 8), y);
  }
  __syncthreads();
  const int c16 = lane % 16, q = lane / 16;
  v4f acc[3] = {};
  {   // a wave to each product of each chunk: its three tiles that have elements on or below the diagonal
    const int r0 = wave / 2 * C;
    const Matrix<P, B, KT * 32>& left = wave % 2 ? u.in.q : u.in.k;
#pragma unroll
    for (int f = 0; f < KT; ++f) {
      const Frag<P> a0 = left.along(r0, f), a1 = left.along(r0 + 16, f);
      const Frag<P> b0 = u.in.k.along(r0, f), b1 = u.in.k.along(r0 + 16, f);
      acc[0] = mma<3>(a0, b0, acc[0]);
      acc[1] = mma<3>(a1, b0, acc[1]);
      acc[2] = mma<3>(a1, b1, acc[2]);
    }
  }
  __syncthreads();
  // the decays, by the lanes that hold the products: P is finished, M and M beta go on
  {
    const int chunk = wave / 2;
    float* out = matrices_of(a, w.index, h, chunk) + C * C;
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = (t ? 16 : 0) + 4 * q + i, c = (t == 2 ? 16 : 0) + c16;
        const float x = power(g[chunk * C + r] - g[chunk * C + c]) * acc[t][i];
        if (wave % 2) {
          out[r * C + c] = r >= c ? a.scale * x : 0.f;
        } else {
          const float m = r > c ? x : 0.f;
          u.m.mat[chunk][1][r][c] = m;
          u.m.mat[chunk][0][r][c] = m * beta[chunk * C + c];
        }
      }
    if (wave % 2)
#pragma unroll
      for (int i = 0; i < 4; ++i) out[(4 * q + i) * C + 16 + c16] = 0.f;
  }
  __syncthreads();
  if (wave == 0) {
    const int chunk = q / 2, o = q % 2 * 16;
    float n[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s[4] = {u.m.mat[chunk][1][o + r][o + c16], 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < r; ++m) s[m % 4] = fmaf(-u.m.mat[chunk][0][o + r][o + m], n[m], s[m % 4]);
      n[r] = (s[0] + s[1]) + (s[2] + s[3]);
      u.m.n[q][r][c16] = n[r];
    }
    float* out = matrices_of(a, w.index, h, chunk);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      out[(o + r) * C + o + c16] = n[r];
      if (o == 0) out[r * C + 16 + c16] = 0.f;
    }
  }
  __syncthreads();
  if (wave < 2) {   // a chunk to each; a result's rows 4 q + i are the next product's contracted index, in that order
    const int chunk = wave;
    v4f x, y;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = u.m.mat[chunk][1][16 + 4 * q + i][c16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x = __builtin_amdgcn_mfma_f32_16x16x4f32(-u.m.mat[chunk][0][16 + c16][4 * q + i], u.m.n[2 * chunk][4 * q + i][c16], x, 0, 0, 0);
    y = x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y = __builtin_amdgcn_mfma_f32_16x16x4f32(-u.m.n[2 * chunk + 1][c16][4 * q + i] * beta[chunk * C + 16 + 4 * q + i], x[i], y, 0, 0, 0);
    float* out = matrices_of(a, w.index, h, chunk);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[(16 + 4 * q + i) * C + c16] = y[i];
  }
}

// ------------------------------------------------------------------ the chain over a sequence's chunks
// What a chunk's waves share, on its way from memory and in LDS. OUT: with Q and P (in PN parts), else K and N alone.
template <class T, int KT, int W, int PN, bool OUT>
struct Chunk {
  static constexpr int P = In<T>::P, UNITS = C * KT * 8, STEP = 64 * W / (KT * 8), PER = (UNITS + 64 * W - 1) / (64 * W);
  static constexpr int FOURS = (OUT ? 2 : 1) * C * C / 4, PAIR = (FOURS + 64 * W - 1) / (64 * W);
  struct Shared {
    Matrix<P, C, KT * 32> k;
    Matrix<OUT ? P : 1, OUT ? C : 1, KT * 32> q;
    Matrix<3, C, C> n;
    Matrix<PN, OUT ? C : 1, C> p;
    alignas(16) float grow[C], rest[C], beta[C], whole;
  };
  Vec<T, 4> k[PER], q[OUT ? PER : 1];
  Vec<float, 4> pair[PAIR];
  float scalar;
  // this thread's first element of K and Q, in bytes from a chunk's, and how many of four there are; the others are STEP rows apart
  unsigned k0, q0;
  int n;
  __device__ __forceinline__ explicit Chunk(const DeltaArgs& a) {
    const int four = threadIdx.x % (KT * 8), row = threadIdx.x / (KT * 8), left = a.dk - 4 * four;
    n = UNITS < 64 * W && (int)threadIdx.x >= UNITS ? 0 : left < 0 ? 0 : left > 4 ? 4 : left;
    const unsigned col = n ? 4 * four : 0, r = n ? row : 0;
    k0 = (r * (unsigned)a.k_stride + col) * (unsigned)sizeof(T);
    q0 = (r * (unsigned)a.q_stride + col) * (unsigned)sizeof(T);
  }
  __device__ __forceinline__ void fetch(const DeltaArgs& a, long row, int count, size_t block, int half, int h, int hk) {
    const T* K = row_of((const T*)a.k, row, a.k_stride) + (size_t)hk * a.dk;
    const T* Q = row_of((const T*)a.q, row, a.q_stride) + (size_t)hk * a.dk;
    const int mine = threadIdx.x / (KT * 8);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool in = count == C || mine + j * STEP < count;   // rows behind the sequence's end are zeros
      k[j] = load_four(past(K + (in ? j * STEP * a.k_stride : 0), in ? k0 : 0u), in ? n : 0, a.fours);
      if (OUT) q[j] = load_four(past(Q + (in ? j * STEP * a.q_stride : 0), in ? q0 : 0u), in ? n : 0, a.fours);
    }
    const float* m = matrices_of(a, block, h, half);
#pragma unroll
    for (int j = 0; j < PAIR; ++j)
      if (FOURS >= 64 * W || (int)threadIdx.x < FOURS) pair[j] = load_vec(past(m + j * 64 * W * 4, threadIdx.x * 16u), 4);
    const float* f = scalars_of(a, block, h);
    const int t = threadIdx.x < 3 * C ? threadIdx.x / C * B + half * C + threadIdx.x % C : 3 * B + half;
    if (threadIdx.x <= 3 * C) scalar = f[t];
  }
  __device__ __forceinline__ void put(Shared& s) const {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (UNITS < 64 * W && (int)threadIdx.x >= UNITS) continue;
      const int row = threadIdx.x / (KT * 8) + j * STEP, four = threadIdx.x % (KT * 8);
      v2u x[P];
      parts4(k[j], x);
      s.k.put(row, four, x);
      if constexpr (OUT) {
        parts4(q[j], x);
        s.q.put(row, four, x);
      }
    }
#pragma unroll
    for (int j = 0; j < PAIR; ++j) {
      const int u = threadIdx.x + j * 64 * W, r = u % (C * C / 4) / (C / 4), four = u % (C / 4);
      if (FOURS < 64 * W && u >= FOURS) continue;
      const float x[4] = {get(pair[j], 0), get(pair[j], 1), get(pair[j], 2), get(pair[j], 3)};
      if (u < C * C / 4) {
        v2u y[3];
        split4<3>(x, y);
        s.n.put(r, four, y);
      } else if constexpr (OUT) {
        v2u y[PN];
        split4<PN>(x, y);
        s.p.put(r, four, y);
      }
    }
    if (threadIdx.x <= 3 * C) s.grow[threadIdx.x] = scalar;   // and rest, beta and whole behind it
  }
};

// Eight of a wave's values in a chunk: rows 4 (lane / 16) + i of its two tiles, column lane % 16 of the wave's.
__device__ __forceinline__ int chunk_row(int k) { return (k / 4) * 16 + 4 * (threadIdx.x % 64 / 16) + k % 4; }
struct Eight {
  v4f t[2];
  __device__ __forceinline__ explicit Eight(const float (&rows)[C]) {
    t[0] = *(const v4f*)&rows[4 * (threadIdx.x % 64 / 16)];
    t[1] = *(const v4f*)&rows[16 + 4 * (threadIdx.x % 64 / 16)];
  }
  __device__ __forceinline__ float operator[](int k) const { return t[k / 4][k % 4]; }
};

template <class T>
struct Rows8 {
  T v[8];
  // `lane`: bytes of row 4 (lane / 16) and the lane's column from p. Rows behind the last are read as the last: what they meet is 0.
  __device__ __forceinline__ void fetch(const T* p, size_t stride, unsigned lane, unsigned column, int count) {
    if (count == C) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = *past(p + ((k / 4) * 16 + k % 4) * stride, lane);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int r = chunk_row(k) < count ? chunk_row(k) : count - 1;
        v[k] = *past(p, ((unsigned)r * (unsigned)stride + column) * (unsigned)sizeof(T));
      }
    }
  }
};

// A state's 16 columns in a wave: element i of tile m is row 16 m + 4 (lane / 16) + i.
template <int KT>
struct State {
  v4f t[2 * KT];
  __device__ __forceinline__ void load(const float* p, int dk, int width, int col) {
    const int r0 = 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) t[m][i] = p && col < width && 16 * m + r0 + i < dk ? p[(size_t)(16 * m + r0 + i) * width + col] : 0.f;
  }
  __device__ __forceinline__ void store(float* p, int dk, int width, int col) const {
    const int r0 = 4 * (threadIdx.x % 64 / 16);
    if (col >= width) return;
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (dk == 32 * KT || 16 * m + r0 + i < dk) *past(p + (16 * m + i) * width, (unsigned)(r0 * width + col) * 4u) = t[m][i];
  }
  // to a tile of 16 columns
  __device__ __forceinline__ void store_tile(float* p, int dk) const {
    const int r0 = 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (dk == 32 * KT || 16 * m + r0 + i < dk) *past(p + (16 * m + i) * 16, (unsigned)(r0 * 16 + threadIdx.x % 16) * 4u) = t[m][i];
  }
  __device__ __forceinline__ void identity(int col) {
    const int r0 = 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) t[m][i] = 16 * m + r0 + i == col ? 1.f : 0.f;
  }
  __device__ __forceinline__ Frag<3> operand(int f) const {
    const float x[8] = {t[2 * f][0], t[2 * f][1], t[2 * f][2], t[2 * f][3], t[2 * f + 1][0], t[2 * f + 1][1], t[2 * f + 1][2], t[2 * f + 1][3]};
    return split8<3>(x);
  }
};

// What a wave of a chain works on: 16 columns of the state, or of the map that a segment is.
struct Columns {
  int c0, col;     // the first, the lane's
  bool map, any;   // of the map; there are columns
  __device__ __forceinline__ Columns(const DeltaArgs& a, int w, bool maps) {
    const int tile = blockIdx.y * w + threadIdx.x / 64, values = (a.dv + 15) / 16;
    map = maps && tile >= values;
    c0 = 16 * (map ? tile - values : tile);
    col = c0 + threadIdx.x % 16;
    any = c0 < (map ? a.dk : a.dv);
  }
};

__device__ __forceinline__ float* front_of(const DeltaArgs& a, size_t slot, int h) { return a.fronts + state_at(a, slot, h); }
__device__ __forceinline__ float* map_of(const DeltaArgs& a, size_t slot, int h) {
  return a.maps + (slot * a.heads + h) * ((size_t)a.dk * a.dk);
}

// OUT: the chain with its outputs, from the states in front of the segments; else the segments' maps, and what they leave of no state.
template <class T, int KT, int W, bool OUT>
__global__ __launch_bounds__(64 * W, OUT ? 2 : 4) void delta_forward_kernel(DeltaArgs a) {
  constexpr int PO = sizeof(T) == 2 ? 2 : 3;   // o is rounded to 16 bits: two parts leave 2^-16 of its terms
  typedef Chunk<T, KT, W, PO, OUT> Ck;
  __shared__ typename Ck::Shared sh[2];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads);
  const size_t segment = blockIdx.x / a.heads;
  const int lane = threadIdx.x % 64, c16 = lane % 16, q = lane / 16;
  Job w;
  if (!OUT && whole_sequences(a)) return;
  if (!find_job(a, segment, w) || (!OUT && w.last)) return;
  const Columns m(a, W, !OUT && !w.first);
  const int col = m.col;
  long b, e;
  span(a, w.s, b, e);
  const long first = first_block(a, w.s) + w.from;
  b += w.from * B;
  if (e > b + (w.to - w.from) * B) e = b + (w.to - w.from) * B;
  State<KT> S;
  if (w.first) S.load(a.h0 ? a.h0 + state_at(a, w.s, h) : nullptr, a.dk, a.dv, col);
  else if (OUT) S.load(front_of(a, w.slot, h), a.dk, a.dv, col);
  else S.identity(m.map ? col : -1);
  const T* V = (const T*)a.v + (size_t)h * a.dv;
  const bool none = m.map || col >= a.dv;   // no values: a map's columns, and those behind the last
  const unsigned vcol = none ? 0 : col, vlane = (4u * q * (unsigned)a.v_stride + vcol) * (unsigned)sizeof(T);
  const int chunks = (int)((e - b + C - 1) / C);
  const auto rows_in = [&](int c) { return e - b - (long)c * C < C ? (int)(e - b - (long)c * C) : C; };
  Ck next(a);
  Rows8<T> vnext;
  const auto fetch = [&](int c) {
    const long row = b + (long)c * C;
    next.fetch(a, row, rows_in(c), (size_t)(first + c / 2), c % 2, h, hk);
    vnext.fetch(V + row * a.v_stride, a.v_stride, vlane, vcol, rows_in(c));
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
    if (OUT && c + 1 < chunks) fetch(c + 1);
    v4f oq[2] = {};
    float x[8], y[8];
    if (m.any) {
      if (OUT && a.carry && c % 2 == 0) S.store_tile(a.carry + a.carry_states + tiles_at(a, (size_t)(first + c / 2), h) + m.c0 * a.dk, a.dk);
      v4f ks[2] = {};
      Frag<In<T>::P> kf[2][2], qf[2][2];
      const auto read = [&](int f) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          kf[f % 2][r] = t.k.along(16 * r, f);
          if constexpr (OUT) qf[f % 2][r] = t.q.along(16 * r, f);
        }
      };
      read(0);
      const Eight grow(t.grow), beta(t.beta);
      const float whole = t.whole;
      Frag<3> nf[2];
#pragma unroll
      for (int f = 0; f < KT; ++f) {
        if (f + 1 < KT) read(f + 1);
        else
#pragma unroll
          for (int r = 0; r < 2; ++r) nf[r] = t.n.along(16 * r, 0);
        on_their_way<OUT>();
        const v4f decayed[2] = {S.t[2 * f] * whole, S.t[2 * f + 1] * whole};
        const Frag<3> op = S.operand(f);
        S.t[2 * f] = decayed[0], S.t[2 * f + 1] = decayed[1];
        mma2<3>(kf[f % 2], op, ks);
        if constexpr (OUT)
#pragma unroll
          for (int r = 0; r < 2; ++r) oq[r] = mma<PO>(op, qf[f % 2][r], oq[r]);
      }
      on_their_way<OUT>();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = (none ? 0.f : widen((OUT ? v : vnext).v[k])) - grow[k] * ks[k / 4][k % 4];
        y[k] = beta[k] * x[k];
      }
      const Frag<3> rb = split8<3>(y);
      v4f nr[2] = {};
      mma2<3>(nf, rb, nr);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] -= nr[k / 4][k % 4];
    }
    if (!OUT && c + 1 < chunks) fetch(c + 1);
    if (m.any) {
      const Eight beta(t.beta), rest(t.rest);
      if (OUT && a.carry) {
        float* E = a.carry + rows_at(a, (size_t)(first + c / 2), h) + (m.c0 * B + c % 2 * C * 16);
#pragma unroll
        for (int k = 0; k < 8; ++k) *past(E + ((k / 4) * 16 + k % 4) * 16, (unsigned)(4 * q * 16 + c16) * 4u) = x[k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] *= beta[k];
        y[k] = rest[k] * x[k];
      }
      if constexpr (OUT) {
        if (a.o) {
          Frag<PO> pf[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) pf[r] = t.p.along(16 * r, 0);
          const Frag<PO> vo = split8<PO>(x);
          T* O = (T*)a.o + row * a.o_stride + (size_t)h * a.dv + m.c0;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            oq[r] = mma<PO>(vo, pf[r], oq[r] * (t.grow[16 * r + c16] * a.scale));
            if (16 * r + c16 < count) {
              const float o[4] = {oq[r][0], oq[r][1], oq[r][2], oq[r][3]};
              store_four(past(O, ((16u * r + c16) * (unsigned)a.o_stride + 4 * q) * (unsigned)sizeof(T)), pack<T>(o), a.dv - m.c0 - 4 * q, a.fours);
            }
          }
        }
      }
      Frag<In<T>::P> kd[2][2];
      kd[0][0] = t.k.down(0, 0), kd[0][1] = t.k.down(1, 0);
      const Frag<3> up = split8<3>(y);
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        if (i + 1 < KT) kd[(i + 1) % 2][0] = t.k.down(2 * i + 2, 0), kd[(i + 1) % 2][1] = t.k.down(2 * i + 3, 0);
        on_their_way<OUT>();
        v4f two[2] = {S.t[2 * i], S.t[2 * i + 1]};
        mma2<3>(kd[i % 2], up, two);
        S.t[2 * i] = two[0], S.t[2 * i + 1] = two[1];
      }
    }
    if (c + 1 < chunks) next.put(sh[(c + 1) & 1]);
    if (OUT) v = vnext;
    __syncthreads();
  }
  if (OUT) {
    if (a.last && w.last) S.store(a.last + state_at(a, w.s, h), a.dk, a.dv, col);
  } else if (m.map) {
    S.store(map_of(a, w.slot, h), a.dk, a.dk, col);
  } else {
    S.store(front_of(a, w.slot + 1, h), a.dk, a.dv, col);
  }
}

// The same for the gradients, from the last chunk to the first: X and the gradients of the states behind the blocks; or the segments'
// maps from the gradient behind them to the one in front.
template <class T, int KT, int W, bool OUT>
__global__ __launch_bounds__(64 * W) void delta_backward_kernel(DeltaArgs a) {
  typedef Chunk<T, KT, W, 3, true> Ck;
  constexpr int P = In<T>::P;
  __shared__ typename Ck::Shared sh[2];
  const int h = blockIdx.x % a.heads, hk = h / (a.heads / a.key_heads);
  const size_t segment = blockIdx.x / a.heads;
  const int lane = threadIdx.x % 64, c16 = lane % 16, q = lane / 16;
  Job w;
  if (!OUT && whole_sequences(a)) return;
  if (!find_job(a, segment, w) || (!OUT && w.first)) return;
  const Columns m(a, W, !OUT && !w.last);
  const int col = m.col;
  long b, e;
  span(a, w.s, b, e);
  const long first = first_block(a, w.s) + w.from;
  b += w.from * B;
  if (e > b + (w.to - w.from) * B) e = b + (w.to - w.from) * B;
  State<KT> S;   // the gradient of the state behind a chunk
  if (w.last) S.load(a.dlast ? a.dlast + state_at(a, w.s, h) : nullptr, a.dk, a.dv, col);
  else if (OUT) S.load(front_of(a, w.slot, h), a.dk, a.dv, col);
  else S.identity(m.map ? col : -1);
  const T* D = (const T*)a.dout + (size_t)h * a.dv;
  const bool none = m.map || col >= a.dv;
  const unsigned dcol = none ? 0 : col, dlane = (4u * q * (unsigned)a.dout_stride + dcol) * (unsigned)sizeof(T);
  const int chunks = (int)((e - b + C - 1) / C);
  const auto rows_in = [&](int c) { return e - b - (long)c * C < C ? (int)(e - b - (long)c * C) : C; };
  Ck next(a);
  Rows8<T> dnext;
  const auto fetch = [&](int c) {
    const long row = b + (long)c * C;
    next.fetch(a, row, rows_in(c), (size_t)(first + c / 2), c % 2, h, hk);
    dnext.fetch(D + row * a.dout_stride, a.dout_stride, dlane, dcol, rows_in(c));
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
    if (OUT && c > 0) fetch(c - 1);
    float x[8], y[8];
    Frag<3> od;
    if (m.any) {
      if (OUT && (c % 2 || c == chunks - 1)) S.store_tile(a.behind + tiles_at(a, (size_t)(first + c / 2), h) + m.c0 * a.dk, a.dk);
      v4f ks[2] = {};
      Frag<P> kf[2][2];
      const auto read = [&](int f) {
#pragma unroll
        for (int r = 0; r < 2; ++r) kf[f % 2][r] = t.k.along(16 * r, f);
      };
      read(0);
      const Eight grow(t.grow), beta(t.beta), rest(t.rest);
      const float whole = t.whole;
      Frag<3> pf[2], nf[2];
#pragma unroll
      for (int f = 0; f < KT; ++f) {
        if (f + 1 < KT) read(f + 1);
        else
#pragma unroll
          for (int r = 0; r < 2; ++r) pf[r] = t.p.down(r, 0);
        on_their_way<OUT>();
        const v4f decayed[2] = {S.t[2 * f] * whole, S.t[2 * f + 1] * whole};
        const Frag<3> op = S.operand(f);
        S.t[2 * f] = decayed[0], S.t[2 * f + 1] = decayed[1];
        mma2<3>(kf[f % 2], op, ks);
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) nf[r] = t.n.down(r, 0);
      on_their_way<OUT>();
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = none ? 0.f : widen((OUT ? d : dnext).v[k]);
      const Frag<P> dop = split8<P>(x);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        ks[k / 4][k % 4] *= rest[k];
        y[k] = a.scale * grow[k] * x[k];
      }
      od = split8<3>(y);
      mma2<3>(pf, dop, ks);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = ks[k / 4][k % 4];
        y[k] = beta[k] * x[k];
      }
      const Frag<3> z = split8<3>(y);
      v4f nz[2] = {};
      mma2<3>(nf, z, nz);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] -= nz[k / 4][k % 4];
    }
    if (!OUT && c > 0) fetch(c - 1);
    if (m.any) {
      const Eight grow(t.grow), beta(t.beta);
      Frag<P> kd[2][2], qd[2][2];
#pragma unroll
      for (int z = 0; z < 2; ++z) kd[0][z] = t.k.down(z, 0), qd[0][z] = t.q.down(z, 0);
      on_their_way<OUT>();
      if (OUT) {
        float* X = a.x + rows_at(a, (size_t)(first + c / 2), h) + (m.c0 * B + c % 2 * C * 16);
#pragma unroll
        for (int k = 0; k < 8; ++k) *past(X + ((k / 4) * 16 + k % 4) * 16, (unsigned)(4 * q * 16 + c16) * 4u) = x[k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = -grow[k] * beta[k] * x[k];
      const Frag<3> down = split8<3>(y);
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        if (i + 1 < KT)
#pragma unroll
          for (int z = 0; z < 2; ++z) kd[(i + 1) % 2][z] = t.k.down(2 * i + 2 + z, 0), qd[(i + 1) % 2][z] = t.q.down(2 * i + 2 + z, 0);
        on_their_way<OUT>();
        v4f two[2] = {S.t[2 * i], S.t[2 * i + 1]};
        mma2<3>(qd[i % 2], od, two);
        mma2<3>(kd[i % 2], down, two);
        S.t[2 * i] = two[0], S.t[2 * i + 1] = two[1];
      }
    }
    if (c > 0) next.put(sh[(c - 1) & 1]);
    if (OUT) d = dnext;
    __syncthreads();
  }
  if (OUT) {
    if (a.dh0 && w.first) S.store(a.dh0 + state_at(a, w.s, h), a.dk, a.dv, col);
  } else if (m.map) {
    S.store(map_of(a, w.slot, h), a.dk, a.dk, col);
  } else {
    S.store(front_of(a, w.slot - 1, h), a.dk, a.dv, col);
  }
}

// From segment to segment: the state in front of the next (backward: the gradient behind the one before) is the map's share of this one's and what
// the segment leaves of no state, which lies there already. 64 columns to a workgroup, whose waves share a map's parts in LDS; the next
// map is on its way meanwhile: 8 us a step for 128 x 128.
template <int KT, bool BACK>
__global__ __launch_bounds__(256) void delta_join_kernel(DeltaArgs a) {
  constexpr int PER = 32 * KT * KT * 8 / 256;
  __shared__ Matrix<3, 32 * KT, 32 * KT> map;
  const int h = blockIdx.x % a.heads;
  if (whole_sequences(a)) return;
  const size_t s = blockIdx.x / a.heads;
  const long size = a.begin ? a.first_segment[a.n_seq + 1] : a.segment, blocks = first_block(a, s + 1) - first_block(a, s);
  const long count = segments_of(blocks, size);
  if (count < 3) return;
  const int col = (blockIdx.y * 4 + threadIdx.x / 64) * 16 + threadIdx.x % 16;
  const size_t base = first_slot(a, s);
  const auto place = [&](long j) { return base + (BACK ? count - 1 - j : j); };
  Vec<float, 4> next[PER];
  const auto fetch = [&](long j) {
    const float* p = map_of(a, place(j), h);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = threadIdx.x + i * 256, row = x / (KT * 8), four = x % (KT * 8), n = row < a.dk ? a.dk - 4 * four : 0;
      next[i] = load_four(past(p, n > 0 ? (unsigned)(row * a.dk + 4 * four) * 4u : 0u), n, a.fours);
    }
  };
  fetch(1);
  State<KT> S;
  S.load(front_of(a, place(1), h), a.dk, a.dv, col);
  for (long j = 1; j + 1 < count; ++j) {
    float* to = front_of(a, place(j + 1), h);
    State<KT> sum;
    sum.load(to, a.dk, a.dv, col);
    __syncthreads();   // the map in front is done with
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = threadIdx.x + i * 256;
      v2u y[3];
      parts4(next[i], y);
      map.put(x / (KT * 8), x % (KT * 8), y);
    }
    __syncthreads();
    if (j + 2 < count) fetch(j + 1);
#pragma unroll
    for (int f = 0; f < KT; ++f) {
      const Frag<3> op = S.operand(f);
#pragma unroll
      for (int i = 0; i < 2 * KT; ++i) sum.t[i] = mma<3>(map.along(16 * i, f), op, sum.t[i]);
    }
    sum.store(to, a.dk, a.dv, col);
    S = sum;
  }
}

// ------------------------------------------------------------------ the gradients of a block
// With W = beta E, Y = beta X, S and S' the state in front of a block and the gradient behind it, D the decays between its rows, and of a key's heads
//   dP = sum of scale D o (dO W^T),  dM = sum of -D o (Y W^T)  (on and below, and below the diagonal),
//   dq = sum of scale e^G dO S^T + dP K,  dk = sum of (e^{G_end - G} W S'^T - e^G Y S^T) + dP^T Q + dM K + dM^T K,  dv = Y.
// A decay's gradient needs no more products: where all of a state is scaled, what o gains is q.dq, and what v would have to gain for
// the errors to follow is v.dv, so that G's gradient at a row is q.dq - v.dv, and at the last the state's own, <S', the state behind>, as well.
// Of q.dq the part of dP is the sum over a row of dP o (Q K^T).
//
// Eight waves, each with 16 columns of dq and dk; the heads that share a key one behind the other, their sums kept in LDS where there
// is room and in the workspace where not (each thread its own; 107 of 500 us where all were in the workspace). Values, their gradients and
// the states pass in steps of 32 columns, the next on its way meanwhile, its operands in the other half of the LDS. What becomes dq and dk alone, which are rounded to the inputs' type, is formed from two parts where that is a type
// of 16 bits (2^-16 of the terms are left out); what becomes ddecay too, in 32 bits, from all. All 256 registers of a lane are in use, and some
// more in scratch: 2 .. 12 for types of 16 bits, 11 .. 51 for those of 32.
template <class T, int KT, int WIDTH>
__global__ __launch_bounds__(512) void delta_gradient_kernel(DeltaArgs a) {
  constexpr int P = In<T>::P, PK = sizeof(T) == 2 ? 2 : 3, LV = 32 + 8, Y = P, W = P + PK, PLANES = P + PK + 3;
  constexpr bool KEEP = P < 3;   // there is room for K beside Q
  typedef bf16 Plane[B][LV];
  struct Rows {
    float dots[8][B], prow[4][B], ends[8];
  };
  struct Pair {
    Matrix<PK, B, B> p, m;
  };
  __shared__ union {
    alignas(16) Plane step[2][PLANES];   // dO, beta X, beta E
    Rows rows;
    Pair pair;
    Matrix<P, B, KT * 32> k;
  } u;
  __shared__ Matrix<P, B, KT * 32> kq;
  __shared__ Matrix<KEEP ? P : 1, KEEP ? B : 1, KT * 32> kept_k;
  __shared__ double g[B];
  __shared__ float grow[B], rest[B], beta[B], vrow[B];
  __shared__ float kept_here[P == 1 ? 28 : 1][512];   // dq's and the pairs' sums, where there is room
  Block w;
  const int hk = blockIdx.x % a.key_heads, group = a.heads / a.key_heads;
  if (!find_block(a, blockIdx.x / a.key_heads, w)) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c16 = lane % 16, q = lane / 16;
  const bool owner = wave < 2 * KT;
  const int kc = 16 * wave + c16;   // the column of dq and dk
  const T* K = row_of((const T*)a.k, w.row, a.k_stride) + (size_t)hk * a.dk;
  const T* Q = row_of((const T*)a.q, w.row, a.q_stride) + (size_t)hk * a.dk;
  const auto load_kq = [&](const T* p, unsigned stride, Matrix<P, B, KT * 32>& to) {
    Vec<T, 4> x[B * KT * 8 / 512];
#pragma unroll
    for (int j = 0; j < B * KT * 8 / 512; ++j) {
      const int i = threadIdx.x + j * 512, row = i / (KT * 8), four = i % (KT * 8), n = row < w.count ? a.dk - four * 4 : 0;
      x[j] = load_four(past(p, n > 0 ? (row * stride + four * 4) * (unsigned)sizeof(T) : 0u), n, WIDTH);
    }
#pragma unroll
    for (int j = 0; j < B * KT * 8 / 512; ++j) {
      const int i = threadIdx.x + j * 512;
      v2u y[P];
      parts4(x[j], y);
      to.put(i / (KT * 8), i % (KT * 8), y);
    }
  };
  // tiles on and below the diagonal: of dO W^T those numbered 0 .. 9, of Y W^T 10 .. 19; a wave has every eighth
  const auto tile_of = [](int o, int& it, int& jt) {
    it = o >= 6 ? 3 : o >= 3 ? 2 : o >= 1 ? 1 : 0;
    jt = o - it * (it + 1) / 2;
  };
  Matrix<P, B, KT * 32>& km = [&]() -> Matrix<P, B, KT * 32>& {
    if constexpr (KEEP) return kept_k;
    else return u.k;
  }();
  const int row = threadIdx.x / 8, col = 4 * (threadIdx.x % 8);
  const bool in = row < w.count;
  const unsigned d_at = (row * (unsigned)a.dout_stride + col) * (unsigned)sizeof(T), v_at = (row * (unsigned)a.v_stride + col) * (unsigned)sizeof(T);
  const unsigned e_at = (unsigned)(col / 16 * (B * 16) + row * 16 + col % 16) * 4u, s_at = (unsigned)(q / 2 * (a.dk * 16) + kc * 16 + q % 2 * 8) * 4u;
  const int tiled = tiled_columns(a);
  Vec<T, 4> d, v;
  Vec<float, 4> ev, xv, s0[2], s1[2];
  const auto fetch = [&](int h, int v0) {
    const int n = in ? a.dv - v0 - col : 0;
    const size_t at = (size_t)h * a.dv + v0;
    d = load_four(past((const T*)a.dout + w.row * a.dout_stride + at, n > 0 ? d_at : 0u), n, WIDTH);
    v = load_four(past((const T*)a.v + w.row * a.v_stride + at, n > 0 ? v_at : 0u), n, WIDTH);
    // a tile's columns are all there, zeros behind the last
    const int rows = in && v0 + col < tiled ? 4 : 0, states = owner && kc < a.dk && v0 + 8 * q < tiled ? 4 : 0;
    ev = load_four(past(a.carry_in + rows_at(a, w.index, h) + v0 * B, rows ? e_at : 0u), rows, FOURS);
    xv = load_four(past(a.x + rows_at(a, w.index, h) + v0 * B, rows ? e_at : 0u), rows, FOURS);
    const float* before = a.carry_in + a.carry_states + tiles_at(a, w.index, h) + v0 * a.dk;
    const float* behind = a.behind + tiles_at(a, w.index, h) + v0 * a.dk;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      s0[k] = load_four(past(before + 4 * k, states ? s_at : 0u), states, FOURS);
      s1[k] = load_four(past(behind + 4 * k, states ? s_at : 0u), states, FOURS);
    }
  };
  // a head's sums of decays and rates, of the row that this thread stands for
  double sum = 0.0, half = 0.0, last = 0.0;
  float rate = 0.f;
  const auto ahead = [&](int h) {
    if (threadIdx.x >= B) return;
    const double* sums = sums_of(a, w.index, h);
    sum = sums[threadIdx.x], half = sums[C - 1], last = sums[B - 1];
    rate = scalars_of(a, w.index, h)[2 * B + threadIdx.x];
  };
  ahead(hk * group);
  fetch(hk * group, 0);
  load_kq(Q, (unsigned)a.q_stride, kq);
  load_kq(K, (unsigned)a.k_stride, km);
  __syncthreads();
  v4f qk[2] = {};   // Q K^T in the wave's tiles of dP
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (wave + 8 * k < 10) {
      int it, jt;
      tile_of(wave + 8 * k, it, jt);
#pragma unroll
      for (int f = 0; f < KT; ++f) qk[k] = mma<3>(kq.along(16 * it, f), km.along(16 * jt, f), qk[k]);
    }
  int turn = 0;
  // the group's sums: dq's and dk's 16 values of this thread each, and dP's and dM's 12
  float* kept = a.kept + ((w.index * a.key_heads + hk) * 44) * 512;
  v4f dq[4], dr[4], dc[4], pair[3];
  for (int h = hk * group; h < (hk + 1) * group; ++h) {
    __syncthreads();   // LDS is free
    if (threadIdx.x < B) {
      const double end = half + last, mine = sum + (threadIdx.x >= C ? half : 0.0);
      g[threadIdx.x] = mine;
      grow[threadIdx.x] = power(mine);
      rest[threadIdx.x] = power(end - mine);
      beta[threadIdx.x] = rate;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) dq[t] = dr[t] = dc[t] = (v4f)0.f;
#pragma unroll
    for (int k = 0; k < 3; ++k) pair[k] = (v4f)0.f;
    float ss = 0.f, dbeta = 0.f, dvv = 0.f;
    __syncthreads();
    for (int v0 = 0; v0 < a.dv; v0 += 32, turn ^= 1) {
      Plane* step = u.step[turn];
      float f0[8], f1[8];
      {
        const int n = in ? a.dv - v0 - col : 0;
        const size_t at = (size_t)h * a.dv + v0;
        const float b = beta[row];
        float y[4], e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          dbeta = fmaf(get(xv, i), get(ev, i), dbeta);
          y[i] = b * get(xv, i);
          e[i] = b * get(ev, i);
          dvv = fmaf(y[i], get(v, i), dvv);
        }
        store_four((T*)a.dvalue + (w.row + row) * a.dv_stride + at + col, pack<T>(y), n, WIDTH);
        v2u x[3], yp[PK], z[P];
        parts4(d, z);
#pragma unroll
        for (int i = 0; i < P; ++i) *(v2u*)&step[i][row][col] = z[i];
        split4<PK>(y, yp);
#pragma unroll
        for (int i = 0; i < PK; ++i) *(v2u*)&step[Y + i][row][col] = yp[i];
        split4<3>(e, x);
#pragma unroll
        for (int i = 0; i < 3; ++i) *(v2u*)&step[W + i][row][col] = x[i];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          f0[k] = get(s0[k / 4], k % 4), f1[k] = get(s1[k / 4], k % 4);
          ss = fmaf(f0[k], f1[k], ss);
        }
      }
      if (v0 + 32 < a.dv) fetch(h, v0 + 32);
      else if (h + 1 < (hk + 1) * group) fetch(h + 1, 0);
      __syncthreads();
      // one part of four tiles of rows after the other, the four side by side
      const auto times = [&](int plane, int parts, int order, const Frag<3>& f, v4f(&c)[4]) {
#pragma unroll
        for (int i = parts - 1; i >= 0; --i) {
          v8bf op[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) op[t] = *(const v8bf*)&step[plane + i][16 * t + c16][8 * q];
#pragma unroll
          for (int j = order - 1 - i; j >= 0; --j)
#pragma unroll
            for (int t = 0; t < 4; ++t) c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[t], __builtin_bit_cast(v8bf, f.p[j]), c[t], 0, 0, 0);
        }
      };
      if (owner) {
        const Frag<3> s = split8<3>(f0);
        times(0, P, 3, s, dq);
        times(Y, PK, PK, s, dr);
        times(W, 3, 3, split8<3>(f1), dc);
      }
      const auto operand = [&](int plane, auto& f, int r0) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(f.p) / sizeof(f.p[0])); ++i) f.p[i] = *(const v4u*)&step[plane + i][r0 + c16][8 * q];
      };
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int t = wave + 8 * k;
        int it, jt;
        tile_of(t % 10, it, jt);
        if (t < 10) {
          Frag<P> l;
          Frag<3> r;
          operand(0, l, 16 * it);
          operand(W, r, 16 * jt);
          pair[k] = mma<3>(l, r, pair[k]);
        } else if (t < 20) {
          Frag<PK> l, r;
          operand(Y, l, 16 * it);
          operand(W, r, 16 * jt);
          pair[k] = mma<PK>(l, r, pair[k]);
        }
      }
    }
    // by row: dbeta and v.dv from the eight threads of one, q.dq from the waves' columns and the tiles of dP. (Addresses of what follows are
    // formed here, from a thread's number that the compiler takes for another in each turn: in front of the loop they would fill the registers.)
    unsigned id = threadIdx.x;
    asm volatile("" : "+v"(id));
    const int lane = id % 64, wave = id / 64, c16 = lane % 16, q = lane / 16, kc = 16 * wave + c16;
    const unsigned mine = id * 4u;
    float kv[KEEP ? 1 : 4][4];
    if constexpr (!KEEP)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // of the last row and column beyond them: what they meet is 0
        const int r = 16 * t + 4 * q + i < w.count ? 16 * t + 4 * q + i : w.count - 1, c = kc < a.dk ? kc : a.dk - 1;
        kv[t][i] = widen(*past(K, ((unsigned)r * (unsigned)a.k_stride + c) * (unsigned)sizeof(T)));
      }
    if (h + 1 < (hk + 1) * group) ahead(h + 1);
    dbeta = group_sum<8>(dbeta), dvv = group_sum<8>(dvv);
    if (threadIdx.x % 8 == 0) {
      if (in) a.dbeta[(w.row + row) * a.dbeta_stride + h] = dbeta;
      vrow[row] = dvv;
    }
    __syncthreads();
    float tail = power(g[B - 1]) * ss;   // <S', the state behind>
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * t + 4 * q + i;
        const float f = grow[r];
        dq[t][i] *= a.scale * f;
        const float c = rest[r] * dc[t][i];
        if constexpr (KEEP) {
          float y = 0.f;
          if (owner)
#pragma unroll
            for (int z = P - 1; z >= 0; --z) y += widen(km.at[z][km.place(r, kc)]);
          tail = fmaf(y, c, tail);
        } else {
          tail = fmaf(kv[t][i], c, tail);
        }
        dr[t][i] = fmaf(-f, dr[t][i], c);   // both of dk's
        float x = 0.f;
        if (owner)
#pragma unroll
          for (int z = P - 1; z >= 0; --z) x += widen(kq.at[z][kq.place(r, kc)]);
        x = sum16(x * dq[t][i]);
        if (c16 == 0) u.rows.dots[wave][r] = x;
      }
    tail = group_sum<64>(tail);
    if (lane == 0) u.rows.ends[wave] = tail;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int t = wave + 8 * k;
      if (t >= 20) continue;
      int it, jt;
      tile_of(t % 10, it, jt);
      const int j = 16 * jt + c16;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * it + 4 * q + i;
        const bool there = t >= 10 ? r > j : r >= j;
        pair[k][i] = there ? (t >= 10 ? -1.f : a.scale) * power(g[r] - g[j]) * pair[k][i] : 0.f;
        if (t < 10) {
          const float y = sum16(pair[k][i] * qk[k < 2 ? k : 0][i]);
          if (c16 == 0) u.rows.prow[jt][r] = y;
        }
      }
    }
    if (group > 1) {   // to the heads in front
      const auto place = [&](int n) { return P == 1 && (n < 16 || n >= 32) ? &kept_here[n < 16 ? n : n - 16][id] : past(kept + n * 512, mine); };
      if (h > hk * group) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) dq[t][i] += *place(4 * t + i), dr[t][i] += *place(16 + 4 * t + i);
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) pair[k][i] += *place(32 + 4 * k + i);
      }
      if (h + 1 < (hk + 1) * group) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) *place(4 * t + i) = dq[t][i], *place(16 + 4 * t + i) = dr[t][i];
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) *place(32 + 4 * k + i) = pair[k][i];
      }
    }
    __syncthreads();
    if (wave == 0) {
      float x = -vrow[lane], end = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) x += u.rows.dots[i][lane], end += u.rows.ends[i];
      for (int i = 0; i <= lane / 16; ++i) x += u.rows.prow[i][lane];
      if (lane == B - 1) x += end;
#pragma unroll
      for (int d = 1; d < B; d *= 2) {
        const float down = __shfl_down(x, d, 64);
        if (lane + d < B) x += down;
      }
      if (lane < w.count) a.ddecay[(w.row + lane) * a.ddecay_stride + h] = x;
    }
  }
  __syncthreads();
  // dP and dM into LDS, with zeros above the diagonal where an operand has them, and their products
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int t = wave + 8 * k, zero = t - 20;   // 20 .. 23: the tiles (0, 1) and (2, 3) of both
    int it, jt;
    tile_of(t % 10, it, jt);
    const int i0 = 16 * (zero >= 0 ? zero / 2 * 2 : it), j = 16 * (zero >= 0 ? zero / 2 * 2 + 1 : jt) + c16;
    float x[4], none[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = zero >= 0 ? 0.f : pair[k][i];
    unsigned p[PK][4];
    split<PK, 4>(x, none, p);
    Matrix<PK, B, B>& m = (zero >= 0 ? zero % 2 : t >= 10) ? u.pair.m : u.pair.p;
#pragma unroll
    for (int z = 0; z < PK; ++z)
#pragma unroll
      for (int i = 0; i < 4; ++i) *(unsigned short*)&m.at[z][m.place(i0 + 4 * q + i, j)] = (unsigned short)p[z][i];
  }
  __syncthreads();
  if (owner)
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const Frag<P> b = kq.down(wave, 32 * f);
#pragma unroll
      for (int t = 0; t < 2 * f + 2; ++t) dr[t] = mma<PK>(u.pair.p.down(t, 32 * f), b, dr[t]);
    }
  if (!KEEP) {
    __syncthreads();
    load_kq(K, (unsigned)a.k_stride, kq);
    __syncthreads();
  }
  if (!owner) return;
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const Frag<P> b = (KEEP ? km : kq).down(wave, 32 * f);
#pragma unroll
    for (int t = 0; t < 2 * f + 2; ++t) dr[t] = mma<PK>(u.pair.m.down(t, 32 * f), b, dr[t]);
#pragma unroll
    for (int t = 2 * f; t < 4; ++t) {
      dq[t] = mma<PK>(u.pair.p.along(16 * t, f), b, dq[t]);
      dr[t] = mma<PK>(u.pair.m.along(16 * t, f), b, dr[t]);
    }
  }
  if (kc >= a.dk) return;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * t + 4 * q + i;
      if (r >= w.count) continue;
      ((T*)a.dq)[(w.row + r) * a.dq_stride + (size_t)hk * a.dk + kc] = (T)dq[t][i];
      ((T*)a.dkey)[(w.row + r) * a.dk_stride + (size_t)hk * a.dk + kc] = (T)dr[t][i];
    }
}

// ------------------------------------------------------------------ one row of every sequence
// Bound by HBM: 48 sequences of 16 heads of 128 x 128, 101 MB, in 18.5 us (5.5 TB/s, part of it from the memory-side cache).
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
  size_t blocks, segments, slots, first, first_segment, first_slot, order, table, matrices, scalars, sums, x, behind, kept, fronts, maps, bytes;   // offsets into the workspace
};
Sizes sizes_of(size_t rows, size_t n, size_t heads, size_t key_heads, size_t dk, size_t dv, bool backward) {
  Sizes s;
  s.blocks = rows / B + (n < rows ? n : rows);
  s.segments = rows / B >= 24 ? s.blocks / DELTA_SEGMENT + n : 0;
  // a sequence of b blocks is cut where b > 8, into at most (b + 7) / 8; it has more than 64 (b - 1) rows, 256 and more for each of those
  s.slots = s.segments ? rows / (B * DELTA_SEGMENT / 2) : 0;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t p = at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  s.first = take((n + 2) * sizeof(int));
  s.first_segment = take((n + 2) * sizeof(int));
  s.first_slot = take(n * sizeof(int));
  s.order = take(n <= DELTA_ORDER ? n * sizeof(int) : 0);
  s.table = take(s.blocks * 2 * sizeof(int));
  s.matrices = take(s.blocks * heads * 4 * C * C * sizeof(float));
  s.scalars = take(s.blocks * heads * 4 * B * sizeof(float));
  s.sums = take(s.blocks * heads * B * sizeof(double));
  const size_t tiled = (dv + 15) / 16 * 16;
  s.x = take(backward ? s.blocks * heads * B * tiled * sizeof(float) : 0);
  s.behind = take(backward ? s.blocks * heads * dk * tiled * sizeof(float) : 0);
  s.kept = take(backward && heads > key_heads ? s.blocks * key_heads * 44 * 512 * sizeof(float) : 0);
  s.fronts = take(s.slots * heads * dk * dv * sizeof(float));
  s.maps = take(s.slots * heads * dk * dk * sizeof(float));
  s.bytes = at;
  return s;
}

// Workgroups that a sequence and head's columns take.
unsigned groups_of(size_t tiles) { return tiles <= 4 ? 1 : (unsigned)((tiles + 7) / 8); }

void lay_out(DeltaArgs& a, bool backward) {
  const Sizes s = sizes_of(a.rows, a.n_seq, a.heads, a.key_heads, a.dk, a.dv, backward);
  char* w = (char*)a.workspace;
  a.fours = a.dk % 4 == 0 && a.dv % 4 == 0 ? FOURS : a.dk >= 4 && a.dv >= 4 ? ROWS : NARROW;
  a.blocks = s.blocks;
  a.segments = s.segments;
  a.slots = s.slots;
  a.first = (int*)(w + s.first);
  a.first_segment = (int*)(w + s.first_segment);
  a.first_slot = (int*)(w + s.first_slot);
  a.order = (int*)(w + s.order);
  a.table = (int*)(w + s.table);
  a.matrices = (float*)(w + s.matrices);
  a.scalars = (float*)(w + s.scalars);
  a.sums = (double*)(w + s.sums);
  a.x = (float*)(w + s.x);
  a.behind = (float*)(w + s.behind);
  a.kept = (float*)(w + s.kept);
  a.fronts = (float*)(w + s.fronts);
  a.maps = (float*)(w + s.maps);
  a.carry_states = s.blocks * a.heads * B * ((a.dv + 15) / 16 * 16);
}

hipError_t plan(DeltaArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  const long work = (long)a.heads * groups_of((a.dv + 15) / 16);
  if (a.begin) {
    e = launch(delta_plan_kernel, dim3(1), dim3(PLAN), 0, stream, a, work);
  } else if (a.segments) {
    const long blocks = blocks_of((long)a.rows);
    a.segment = segment_blocks(blocks, blocks, work);
    a.segments = a.n_seq && blocks > a.segment ? (size_t)segments_of(blocks, a.segment) : 0;
  }
  const size_t groups = (a.rows + 3) / 4;
  if (e == hipSuccess && a.zero_others && a.rows && (a.begin || !a.n_seq))
    e = launch(delta_zero_kernel, dim3((unsigned)(groups < 2048 ? groups : 2048)), dim3(256), 0, stream, a);
  return e;
}

template <class T, int KT>
hipError_t prepare(const DeltaArgs& a, hipStream_t stream) {
  return launch(delta_prepare_kernel<T, KT>, dim3((unsigned)(a.blocks * a.heads)), dim3(256), 0, stream, a);
}

// The chain: where sequences may be long, the segments' maps and their join in front of it.
template <class T, int KT, int W, bool BACK>
hipError_t chain(const DeltaArgs& a, hipStream_t stream) {
  const unsigned x = (unsigned)((a.segments ? a.segments : a.n_seq) * a.heads), values = (a.dv + 15) / 16, keys = (a.dk + 15) / 16;
  const auto groups = [](unsigned tiles) { return (tiles + W - 1) / W; };
  hipError_t e = hipSuccess;
  if (a.segments) {
    if constexpr (BACK) e = launch(delta_backward_kernel<T, KT, W, false>, dim3(x, groups(values + keys)), dim3(64 * W), 0, stream, a);
    else e = launch(delta_forward_kernel<T, KT, W, false>, dim3(x, groups(values + keys)), dim3(64 * W), 0, stream, a);
    if (e == hipSuccess)
      e = launch(delta_join_kernel<KT, BACK>, dim3((unsigned)(a.n_seq * a.heads), (a.dv + 63) / 64), dim3(256), 0, stream, a);
  }
  if (e != hipSuccess) return e;
  if constexpr (BACK) return launch(delta_backward_kernel<T, KT, W, true>, dim3(x, groups(values)), dim3(64 * W), 0, stream, a);
  else return launch(delta_forward_kernel<T, KT, W, true>, dim3(x, groups(values)), dim3(64 * W), 0, stream, a);
}

// Whether a sequence and head's columns go to workgroups of four waves instead of eight: where four have them all, and where types of several
// parts, whose waves do more, leave half of the compute units without a workgroup of eight (8 sequences of 1,024 rows, 8 heads of 128 x
// 128, either direction: f32 238 us in eights, 178 in fours, fp16 184 and 154, bf16 152 and 159; with 24 sequences and 16 heads bf16 300 and 400).
template <class T>
bool in_fours(const DeltaArgs& a) {
  const size_t eights = a.n_seq * a.heads * ((a.dv + 127) / 128);
  return a.dv <= 64 || (In<T>::P > 1 && eights <= 128 && a.rows / B < 24 * a.n_seq);
}

template <class T, int KT>
hipError_t forward(const DeltaArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.blocks) e = prepare<T, KT>(a, stream);
  if (e != hipSuccess || !a.n_seq) return e;
  return in_fours<T>(a) ? chain<T, KT, 4, false>(a, stream) : chain<T, KT, 8, false>(a, stream);
}

template <class T, int KT>
hipError_t backward(const DeltaArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.blocks) e = prepare<T, KT>(a, stream);
  if (e != hipSuccess || !a.n_seq) return e;
  e = in_fours<T>(a) ? chain<T, KT, 4, true>(a, stream) : chain<T, KT, 8, true>(a, stream);
  if (e != hipSuccess || !a.blocks) return e;
  const dim3 grid((unsigned)(a.blocks * a.key_heads));
  if (a.fours == FOURS) return launch(delta_gradient_kernel<T, KT, FOURS>, grid, dim3(512), 0, stream, a);
  if (a.fours == ROWS) return launch(delta_gradient_kernel<T, KT, ROWS>, grid, dim3(512), 0, stream, a);
  return launch(delta_gradient_kernel<T, KT, NARROW>, grid, dim3(512), 0, stream, a);
}

#define BY_KEY(CALL)                  \
  if (a.dk <= 32) return CALL(1);     \
  if (a.dk <= 64) return CALL(2);     \
  return CALL(4);

}  // namespace

extern "C" size_t amp_delta_blocks(size_t rows, size_t n) { return sizes_of(rows, n, 1, 1, 1, 1, false).blocks; }
extern "C" size_t amp_delta_workspace_bytes(size_t rows, size_t n, size_t heads, size_t key_heads, size_t dk, size_t dv, int backward) {
  return sizes_of(rows, n, heads, key_heads, dk, dv, backward).bytes;
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
