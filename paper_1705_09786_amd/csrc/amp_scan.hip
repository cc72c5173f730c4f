// Gated linear recurrence over packed sequences, forward, backward and for single rows (include/amp.h has the formulas).
//
// The rows are cut into tiles of TILE rows by 64 features, whatever sequences they hold: a tile's rows compose to one map
// h -> P h + Q per feature, and maps compose, so that tiles need not wait for each other's rows.  A row that begins a sequence
// takes in h0 and is a cut: its map ignores what comes in (P = -0, which no product of the keeps 1 - z >= 0 gives), so that what
// stands in another sequence, infinities and NaN included, never reaches it.
#include "amp_ops.hip.h"
#include "amp_common.hip.h"

namespace {

constexpr int TPB = 256, TILE = 128, CH = 64;

template <class T>
struct Lay {
  static constexpr int V = Vec<T>::N, LANES = CH / V, TG = TPB / LANES, LS = TILE / TG;
};

constexpr unsigned CUT = 0x80000000u;
enum { FIRST = 1, LAST = 2, VALID = 4 };

__device__ __forceinline__ bool is_cut(float p) { return __float_as_uint(p) == CUT; }
__device__ __forceinline__ float apply(float p, float q, float h) { return is_cut(p) ? q : fmaf(p, h, q); }
// (p, q) then becomes the map of (p, q) followed by (p2, q2).
__device__ __forceinline__ void compose(float& p, float& q, float p2, float q2) {
  q = apply(p2, q2, q);
  p = is_cut(p2) ? p2 : p * p2;
}

// z = 1 / (1 + e^-g) and keep = 1 - z, both exact to the last bits however near to 0 they are; 0 and 1 at infinite g.
__device__ __forceinline__ void gate_of(float g, float& z, float& keep) {
  const float s = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(g)), r = __builtin_amdgcn_rcpf(1.f + s), small = s * r;
  z = g >= 0.f ? r : small;
  keep = g >= 0.f ? small : r;
}

__device__ __forceinline__ long bound_at(const void* p, int bytes, size_t s, long lo, long hi) {
  const long v = bytes == 8 ? ((const long*)p)[s] : (long)((const int*)p)[s];
  return v < lo ? lo : v > hi ? hi : v;
}

struct TileRows {
  int seq[TILE];              // the sequence of a row, where it has one
  unsigned char flag[TILE];   // FIRST, LAST, VALID
  int part[TPB / 64];
};

// Fills in the tile's rows.  Returns the sequences [s0, s1) that begin in the tile; those behind the last row belong to the last
// tile.  Sorted bounds give every row its sequence; unsorted ones give it some sequence, and no access leaves its array.
template <class A>
__device__ __forceinline__ void tile_rows(const A& a, long t0, TileRows& t, size_t& s0, size_t& s1) {
  const long rows = (long)a.rows, t1 = t0 + TILE;
  const int i = threadIdx.x;
  if (!a.begin) {
    if (i < TILE) {
      t.seq[i] = 0;
      t.flag[i] = t0 + i < rows ? VALID | (t0 + i == 0 ? FIRST : 0) | (t0 + i == rows - 1 ? LAST : 0) : 0;
    }
    s0 = 0;
    s1 = t0 == 0;
    __syncthreads();
    return;
  }
  size_t lo = 0, hi = t0 > 0 ? a.n_seq : 0;   // the number of sequences that begin in front of t0 is in lo .. hi
  while (lo < hi) {
    const size_t step = (hi - lo + TPB - 1) / TPB, at = lo + i * step;
    const size_t c = __syncthreads_count(at < hi && bound_at(a.begin, a.index_bytes, at, 0, rows) < t0);
    const size_t to = lo + c * step;
    lo = c ? to - step + 1 : lo;
    hi = to < hi ? to : hi;
  }
  s0 = s1 = lo;
  if (i < TILE) t.seq[i] = i == 0 ? (int)lo - 1 : -1;
  __syncthreads();
  for (;; s1 += TPB) {
    const size_t s = s1 + i;
    bool in = s < a.n_seq;
    if (in) {
      const long b = bound_at(a.begin, a.index_bytes, s, 0, rows);
      in = b < t1 || t1 >= rows;
      if (b >= t0 && b < t1 && b < rows) atomicMax(&t.seq[b - t0], (int)s);
    }
    const int c = __syncthreads_count(in);
    if (c < TPB) {
      s1 += c;
      break;
    }
  }
  // every row's sequence: the last one that begins at or in front of it
  int s = i < TILE ? t.seq[i] : -1;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(s, d, 64);
    if ((i & 63) >= d && o > s) s = o;
  }
  if ((i & 63) == 63) t.part[i >> 6] = s;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < TILE / 64; ++w)
    if (w < (i >> 6) && t.part[w] > s) s = t.part[w];
  if (i < TILE) {
    int f = 0;
    if (s >= 0 && t0 + i < rows) {
      const long b = bound_at(a.begin, a.index_bytes, s, 0, rows), e = bound_at(a.end, a.index_bytes, s, b, rows), r = t0 + i;
      if (r >= b && r < e) f = VALID | (r == b ? FIRST : 0) | (r == e - 1 ? LAST : 0);
    }
    t.seq[i] = s;
    t.flag[i] = f;
  }
  __syncthreads();
}

// A thread's rows and features.
template <class T>
struct Place {
  int lane, grp;
  long row;       // its first row in the array, row - t0 = grp * LS
  size_t ch;      // its first feature
  long n;         // features from there on
  __device__ Place(long t0, size_t c0, size_t hidden) {
    lane = threadIdx.x % Lay<T>::LANES;
    grp = threadIdx.x / Lay<T>::LANES;
    row = t0 + grp * Lay<T>::LS;
    ch = c0 + lane * Lay<T>::V;
    n = (long)hidden - (long)ch;
  }
};

template <class T>
__device__ __forceinline__ void load_rows(const void* p, size_t stride, const Place<T>& at, long rows, Vec<T> (&v)[Lay<T>::LS]) {
#pragma unroll
  for (int i = 0; i < Lay<T>::LS; ++i) {
    const long r = at.row + i;
    v[i] = load_vec(row_of((const T*)p, r < rows ? r : 0, stride) + (at.n > 0 ? at.ch : 0), r < rows ? at.n : 0);
  }
}

__device__ __forceinline__ float state_at(const float* p, int seq, size_t hidden, size_t ch, long n) {
  return p && n > 0 ? p[(size_t)seq * hidden + ch] : 0.f;
}

// The maps of a thread's rows, forward: keep h + z v, cuts taking in h0.
template <class T, bool TANH>
__device__ __forceinline__ void row_maps(const ScanArgs& a, const TileRows& t, const Place<T>& at, const Vec<T> (&g)[Lay<T>::LS],
                                         const Vec<T> (&c)[Lay<T>::LS], float (&p)[Lay<T>::LS][Lay<T>::V],
                                         float (&q)[Lay<T>::LS][Lay<T>::V]) {
#pragma unroll
  for (int i = 0; i < Lay<T>::LS; ++i) {
    const int r = at.grp * Lay<T>::LS + i, f = t.flag[r];
#pragma unroll
    for (int k = 0; k < Lay<T>::V; ++k) {
      float z, v = get(c[i], k);
      gate_of(get(g[i], k), z, p[i][k]);
      if (TANH) v = tanh_(v);
      q[i][k] = z * v;
      if (f != VALID) {
        if (f & FIRST) q[i][k] = fmaf(p[i][k], state_at(a.h0, t.seq[r], a.hidden, at.ch + k, at.n - k), q[i][k]);
        if (!(f & VALID)) q[i][k] = 0.f;
        if ((f & FIRST) || !(f & VALID)) p[i][k] = __uint_as_float(CUT);
      }
    }
  }
}

// Per feature, the map of every thread's rows in front of its own (BACK: behind) inside the tile, and the tile's: through LDS, a
// quarter of the row groups to a wave, a feature to a lane.
template <int TG>
struct Maps {
  float p[TG][CH], q[TG][CH], tp[4][CH], tq[4][CH];
};
template <class T, bool BACK>
__device__ __forceinline__ void scan_groups(Maps<Lay<T>::TG>& m, const Place<T>& at, const float (&p)[Lay<T>::V], const float (&q)[Lay<T>::V]) {
  constexpr int V = Lay<T>::V, TG = Lay<T>::TG;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    m.p[at.grp][at.lane * V + k] = p[k];
    m.q[at.grp][at.lane * V + k] = q[k];
  }
  __syncthreads();
  const int quarter = threadIdx.x / CH, c = threadIdx.x % CH;
  float cp = 1.f, cq = 0.f;
#pragma unroll
  for (int i = 0; i < TG / 4; ++i) {
    const int g = quarter * (TG / 4) + (BACK ? TG / 4 - 1 - i : i);
    const float gp = m.p[g][c], gq = m.q[g][c];
    m.p[g][c] = cp;
    m.q[g][c] = cq;
    compose(cp, cq, gp, gq);
  }
  m.tp[quarter][c] = cp;
  m.tq[quarter][c] = cq;
  __syncthreads();
}
// What comes into a thread's rows where x comes into the tile.
template <class T, bool BACK>
__device__ __forceinline__ float into_group(const Maps<Lay<T>::TG>& m, const Place<T>& at, int k, float x) {
  constexpr int TG = Lay<T>::TG;
  const int quarter = at.grp / (TG / 4), c = at.lane * Lay<T>::V + k;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int w = BACK ? 3 - i : i;
    if (BACK ? w > quarter : w < quarter) x = apply(m.tp[w][c], m.tq[w][c], x);
  }
  return apply(m.p[at.grp][c], m.q[at.grp][c], x);
}
template <class T, bool BACK>
__device__ __forceinline__ void tile_map(const Maps<Lay<T>::TG>& m, int c, float& p, float& q) {
  p = 1.f, q = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) compose(p, q, m.tp[BACK ? 3 - i : i][c], m.tq[BACK ? 3 - i : i][c]);
}

// Workspace: the tiles' maps, P and Q, tiles x hidden each; Q's place then holds what comes into each tile.
__device__ __forceinline__ float* ws_p(const ScanArgs& a) { return (float*)a.workspace; }
__device__ __forceinline__ float* ws_q(const ScanArgs& a, size_t tiles) { return (float*)a.workspace + tiles * a.hidden; }

template <class T, bool TANH, bool WRITE>
__global__ __launch_bounds__(TPB) void scan_forward_kernel(ScanArgs a, size_t tiles) {
  typedef Lay<T> L;
  __shared__ TileRows t;
  __shared__ Maps<L::TG> m;
  const long t0 = (long)blockIdx.x * TILE;
  const size_t c0 = (size_t)blockIdx.y * CH;
  const Place<T> at(t0, c0, a.hidden);
  Vec<T> g[L::LS], c[L::LS];
  load_rows<T>(a.gate, a.gate_stride, at, (long)a.rows, g);
  load_rows<T>(a.cand, a.cand_stride, at, (long)a.rows, c);
  size_t s0, s1;
  tile_rows(a, t0, t, s0, s1);
  float p[L::LS][L::V], q[L::LS][L::V];
  row_maps<T, TANH>(a, t, at, g, c, p, q);
  float gp[L::V], gq[L::V];
#pragma unroll
  for (int k = 0; k < L::V; ++k) {
    gp[k] = 1.f, gq[k] = 0.f;
#pragma unroll
    for (int i = 0; i < L::LS; ++i) compose(gp[k], gq[k], p[i][k], q[i][k]);
  }
  scan_groups<T, false>(m, at, gp, gq);
  if (!WRITE) {
    const size_t ch = c0 + threadIdx.x;
    if (threadIdx.x < CH && ch < a.hidden) {
      float tp, tq;
      tile_map<T, false>(m, threadIdx.x, tp, tq);
      ws_p(a)[(size_t)blockIdx.x * a.hidden + ch] = tp;
      ws_q(a, tiles)[(size_t)blockIdx.x * a.hidden + ch] = tq;
    }
    return;
  }
  float h[L::V];
#pragma unroll
  for (int k = 0; k < L::V; ++k) h[k] = into_group<T, false>(m, at, k, at.n > k ? ws_q(a, tiles)[(size_t)blockIdx.x * a.hidden + at.ch + k] : 0.f);
#pragma unroll
  for (int i = 0; i < L::LS; ++i) {
    const int r = at.grp * L::LS + i, f = t.flag[r];
#pragma unroll
    for (int k = 0; k < L::V; ++k) h[k] = apply(p[i][k], q[i][k], h[k]);
    if (a.h && (f & VALID)) store_vec(row_of((T*)a.h, at.row + i, a.h_stride) + (at.n > 0 ? at.ch : 0), pack<T>(h), at.n > 0 ? at.n : 0);
    if (a.last && (f & LAST))
#pragma unroll
      for (int k = 0; k < L::V; ++k)
        if (k < at.n) a.last[(size_t)t.seq[r] * a.hidden + at.ch + k] = h[k];
  }
  if (a.carry && threadIdx.x < CH && c0 + threadIdx.x < a.hidden)
    a.carry[(size_t)blockIdx.x * a.hidden + c0 + threadIdx.x] = ws_q(a, tiles)[(size_t)blockIdx.x * a.hidden + c0 + threadIdx.x];
  // sequences without rows keep h0
  if (a.last && a.last != a.h0)
    for (size_t s = s0 + threadIdx.x; s < s1; s += TPB) {
      const long b = a.begin ? bound_at(a.begin, a.index_bytes, s, 0, (long)a.rows) : 0;
      const long e = a.begin ? bound_at(a.end, a.index_bytes, s, b, (long)a.rows) : (long)a.rows;
      if (e <= b)
        for (size_t ch = c0; ch < c0 + CH && ch < a.hidden; ++ch) a.last[s * a.hidden + ch] = a.h0 ? a.h0[s * a.hidden + ch] : 0.f;
    }
}

// The tiles' maps in turn, a feature to a lane.
template <bool BACK>
__global__ __launch_bounds__(64) void scan_carry_kernel(ScanArgs a, size_t tiles) {
  const size_t ch = (size_t)blockIdx.x * 64 + threadIdx.x;
  if (ch >= a.hidden) return;
  float x = 0.f;
  for (size_t i = 0; i < tiles; ++i) {
    const size_t k = (BACK ? tiles - 1 - i : i) * a.hidden + ch;
    const float p = ws_p(a)[k], q = ws_q(a, tiles)[k];
    ws_q(a, tiles)[k] = x;
    x = apply(p, q, x);
  }
}

// Backward: X_t = keep_t G_t is what a row hands to the row in front of it, G_t = d_t + X_{t+1}, d_t = dh_t (+ dlast at a last
// row); a first row hands it to dh0 and nothing to the row in front, so the cuts are the forward pass's.  h_{t-1} is formed again
// from the tile's carry in 32 bits: that costs no more than reading the rounded h back, and no rounding.
template <class T, bool TANH, bool WRITE>
__global__ __launch_bounds__(TPB) void scan_backward_kernel(ScanArgs a, size_t tiles) {
  typedef Lay<T> L;
  __shared__ TileRows t;
  __shared__ Maps<L::TG> m;
  const long t0 = (long)blockIdx.x * TILE;
  const size_t c0 = (size_t)blockIdx.y * CH;
  const Place<T> at(t0, c0, a.hidden);
  Vec<T> g[L::LS], c[L::LS], d[L::LS];
  load_rows<T>(a.gate, a.gate_stride, at, (long)a.rows, g);
  load_rows<T>(a.cand, a.cand_stride, at, (long)a.rows, c);
  load_rows<T>(a.dh, a.dh_stride, at, (long)a.rows, d);
  size_t s0, s1;
  tile_rows(a, t0, t, s0, s1);
  float p[L::LS][L::V], q[L::LS][L::V], hp[L::LS][L::V], gp[L::V], gq[L::V];
  row_maps<T, TANH>(a, t, at, g, c, p, q);
  if (WRITE) {   // h_{t-1}
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      gp[k] = 1.f, gq[k] = 0.f;
#pragma unroll
      for (int i = 0; i < L::LS; ++i) compose(gp[k], gq[k], p[i][k], q[i][k]);
    }
    scan_groups<T, false>(m, at, gp, gq);
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      float h = into_group<T, false>(m, at, k, k < at.n ? a.carry_in[(size_t)blockIdx.x * a.hidden + at.ch + k] : 0.f);
#pragma unroll
      for (int i = 0; i < L::LS; ++i) {
        const int r = at.grp * L::LS + i;
        hp[i][k] = (t.flag[r] & FIRST) ? state_at(a.h0, t.seq[r], a.hidden, at.ch + k, at.n - k) : h;
        h = apply(p[i][k], q[i][k], h);
      }
    }
    __syncthreads();   // the maps are written again below
  }
  // the maps of X, and d in q's place
#pragma unroll
  for (int k = 0; k < L::V; ++k) {
    gp[k] = 1.f, gq[k] = 0.f;
#pragma unroll
    for (int i = L::LS - 1; i >= 0; --i) {
      const int r = at.grp * L::LS + i, f = t.flag[r];
      q[i][k] = get(d[i], k);
      if (f & LAST) q[i][k] += state_at(a.dlast, t.seq[r], a.hidden, at.ch + k, at.n - k);
      compose(gp[k], gq[k], p[i][k], is_cut(p[i][k]) ? 0.f : p[i][k] * q[i][k]);
    }
  }
  scan_groups<T, true>(m, at, gp, gq);
  if (!WRITE) {
    const size_t ch = c0 + threadIdx.x;
    if (threadIdx.x < CH && ch < a.hidden) {
      float tp, tq;
      tile_map<T, true>(m, threadIdx.x, tp, tq);
      ws_p(a)[(size_t)blockIdx.x * a.hidden + ch] = tp;
      ws_q(a, tiles)[(size_t)blockIdx.x * a.hidden + ch] = tq;
    }
    return;
  }
  float x[L::V];
#pragma unroll
  for (int k = 0; k < L::V; ++k) x[k] = into_group<T, true>(m, at, k, k < at.n ? ws_q(a, tiles)[(size_t)blockIdx.x * a.hidden + at.ch + k] : 0.f);
#pragma unroll
  for (int i = L::LS - 1; i >= 0; --i) {
    const int r = at.grp * L::LS + i, f = t.flag[r];
    float og[L::V], oc[L::V], into[L::V];
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      float z, keep, v = get(c[i], k);
      gate_of(get(g[i], k), z, keep);
      if (TANH) v = tanh_(v);
      const float G = q[i][k] + x[k];
      og[k] = G * (z * keep) * (v - hp[i][k]);
      oc[k] = G * z * (TANH ? fmaf(-v, v, 1.f) : 1.f);
      into[k] = keep * G;
      x[k] = is_cut(p[i][k]) ? 0.f : into[k];
    }
    if (f & VALID) {
      const long n = at.n > 0 ? at.n : 0;
      const size_t ch = at.n > 0 ? at.ch : 0;
      store_vec(row_of((T*)a.dgate, at.row + i, a.dgate_stride) + ch, pack<T>(og), n);
      store_vec(row_of((T*)a.dcand, at.row + i, a.dcand_stride) + ch, pack<T>(oc), n);
      if ((f & FIRST) && a.dh0)
#pragma unroll
        for (int k = 0; k < L::V; ++k)
          if (k < at.n) a.dh0[(size_t)t.seq[r] * a.hidden + at.ch + k] = into[k];
    }
  }
  if (a.dh0 && a.dh0 != a.dlast)
    for (size_t s = s0 + threadIdx.x; s < s1; s += TPB) {
      const long b = a.begin ? bound_at(a.begin, a.index_bytes, s, 0, (long)a.rows) : 0;
      const long e = a.begin ? bound_at(a.end, a.index_bytes, s, b, (long)a.rows) : (long)a.rows;
      if (e <= b)
        for (size_t ch = c0; ch < c0 + CH && ch < a.hidden; ++ch) a.dh0[s * a.hidden + ch] = a.dlast ? a.dlast[s * a.hidden + ch] : 0.f;
    }
}

// One row of every sequence: bound by the call itself.  A group of 16 bytes of the inputs to a lane.
template <class T, bool TANH>
__global__ __launch_bounds__(TPB) void scan_step_kernel(ScanStepArgs a) {
  constexpr int V = Vec<T>::N;
  const size_t per = (a.hidden + V - 1) / V, total = a.rows * per;
  for (size_t i = (size_t)blockIdx.x * TPB + threadIdx.x; i < total; i += (size_t)gridDim.x * TPB) {
    const size_t r = i / per, ch = (i - r * per) * V;
    const long n = (long)(a.hidden - ch);
    const Vec<T> g = load_vec(row_of((const T*)a.gate, r, a.gate_stride) + ch, n);
    const Vec<T> c = load_vec(row_of((const T*)a.cand, r, a.cand_stride) + ch, n);
    float* st = a.state + r * a.state_stride + ch;
    Vec<float> s[V / 4];
    float h[V];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) s[j] = load_vec(st + 4 * j, n - 4 * j);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float z, keep, v = get(c, k);
      gate_of(get(g, k), z, keep);
      if (TANH) v = tanh_(v);
      h[k] = fmaf(keep, get(s[k / 4], k % 4), z * v);
    }
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const float o[4] = {h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]};
      store_vec(st + 4 * j, pack<float>(o), n - 4 * j);
    }
    if (a.h) store_vec(row_of((T*)a.h, r, a.h_stride) + ch, pack<T>(h), n);
  }
}

size_t tiles_of(size_t rows) { return rows ? (rows + TILE - 1) / TILE : 1; }   // sequences without rows have a tile too

}  // namespace

extern "C" size_t amp_scan_carry_rows(int, size_t rows, size_t) { return tiles_of(rows); }
extern "C" size_t amp_scan_workspace_bytes(int, size_t rows, size_t hidden) { return (tiles_of(rows) * hidden * 8 + 15) / 16 * 16; }

#define BY_TANH(K, ...)                                                        \
  if (tanh) {                                                                  \
    if ((e = launch(K<T, true __VA_OPT__(, ) __VA_ARGS__>, grid, dim3(TPB), 0, stream, *a, tiles)) != hipSuccess) return e;  \
  } else {                                                                     \
    if ((e = launch(K<T, false __VA_OPT__(, ) __VA_ARGS__>, grid, dim3(TPB), 0, stream, *a, tiles)) != hipSuccess) return e; \
  }

extern "C" hipError_t amp_scan_forward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream) {
  const size_t tiles = tiles_of(a->rows);
  const dim3 grid((unsigned)tiles, (unsigned)((a->hidden + CH - 1) / CH));
  hipError_t e;
  OPS_BY_TYPE(dtype, BY_TANH(scan_forward_kernel, false));
  if ((e = launch(scan_carry_kernel<false>, dim3((unsigned)((a->hidden + 63) / 64)), dim3(64), 0, stream, *a, tiles)) != hipSuccess) return e;
  OPS_BY_TYPE(dtype, BY_TANH(scan_forward_kernel, true));
  return hipSuccess;
}

extern "C" hipError_t amp_scan_backward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream) {
  const size_t tiles = tiles_of(a->rows);
  const dim3 grid((unsigned)tiles, (unsigned)((a->hidden + CH - 1) / CH));
  hipError_t e;
  OPS_BY_TYPE(dtype, BY_TANH(scan_backward_kernel, false));
  if ((e = launch(scan_carry_kernel<true>, dim3((unsigned)((a->hidden + 63) / 64)), dim3(64), 0, stream, *a, tiles)) != hipSuccess) return e;
  OPS_BY_TYPE(dtype, BY_TANH(scan_backward_kernel, true));
  return hipSuccess;
}

extern "C" hipError_t amp_scan_step_launch(int dtype, int tanh, const ScanStepArgs* a, hipStream_t stream) {
  const size_t v = dtype == 0 ? 4 : 8, blocks = (a->rows * ((a->hidden + v - 1) / v) + TPB - 1) / TPB;
  const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
  OPS_BY_TYPE(dtype, return tanh ? launch(scan_step_kernel<T, true>, grid, dim3(TPB), 0, stream, *a)
                                 : launch(scan_step_kernel<T, false>, grid, dim3(TPB), 0, stream, *a));
}
