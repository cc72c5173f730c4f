// Gated linear recurrence over packed sequences, forward, backward and for single rows (include/amp.h has the formulas).
//
// The rows are cut into tiles of TILE rows by 64 features, whatever sequences they hold: a tile's rows compose to one map
// h -> P h + Q per feature, and maps compose, so that tiles need not wait for each other's rows.  A row that begins a sequence
// takes in h0 and is a cut: its map ignores what comes in (P = -0, which no product of the keeps 1 - z >= 0 gives), so that what
// stands in another sequence, infinities and NaN included, never reaches it.
//
// One pass over the data: a workgroup reads a tile once, publishes its map as one 64-bit word per feature, finds the state that
// comes in from the words of the tiles in front, and writes its rows.  A word is {P, Q}; once the state behind the tile is known it
// is replaced by the map that gives it, {cut, state}, so a reader goes back to the nearest cut.  Four tiles share a second word in
// the same way, and the chain of the states runs over those.  States are formed from the same maps in the same order whichever word a
// reader met: results do not depend on timing.
//
// What bounds it: HBM where rows are long, 805 MB at 4.4 TB/s for 65,536 x 2,048 bf16 forward (184 us; a large copy runs at 5.2 TB/s),
// 1.06 GB at 3.9 TB/s for 41,000 x 2,560 bf16 backward (275 us), whose five arrays of a tile leave room for two workgroups on a
// compute unit, where the forward pass has four.  Where features are few, the chain of the states (hand_over).
#include "amp_ops.hip.h"
#include "amp_common.hip.h"

namespace {

constexpr int TPB = 256, TILE = 128, CARRY = TILE;   // the forward pass leaves the state in front of every tile for the backward pass

// A tile of TILE rows and CH features in a workgroup: V features of a row to a lane, LS rows one behind the other.  V is four in every
// type: 8-byte groups of 16-bit elements have half the maps to join inside a tile that 16-byte groups have (65,536 x 2,048 bf16,
// forward: 221 us with groups of 16 bytes, 187 with these), and 64 features of 16 bits are whole cache lines still.
template <class T, bool NARROW_>
struct Lay {
  typedef T E;
  static constexpr bool NARROW = NARROW_;   // rows shorter than V
  static constexpr int V = 4, CH = 64, LANES = CH / V, TG = TPB / LANES, LS = TILE / TG, PARTS = TPB / CH;
  static_assert(LS % 4 == 0 && TG % PARTS == 0 && CH == 64, "flags by words, a slot to a lane of one wave");
};

constexpr unsigned CUT = 0x80000000u;
enum { FIRST = 1, LAST = 2, VALID = 4, ZERO = 8 };   // ZERO: a row of no sequence whose outputs are to be zeros

__device__ __forceinline__ bool is_cut(float p) { return __float_as_uint(p) == CUT; }
__device__ __forceinline__ float apply(float p, float q, float h) { return is_cut(p) ? q : fmaf(p, h, q); }
// (p, q) then becomes the map of (p, q) followed by (p2, q2).  A cut stays one whatever follows it: p * p2 would not where p2 is no number.
__device__ __forceinline__ void compose(float& p, float& q, float p2, float q2) {
  q = apply(p2, q2, q);
  p = is_cut(p) || is_cut(p2) ? __uint_as_float(CUT) : p * p2;
}

// z = 1 / (1 + e^-g) and keep = 1 - z, both exact to the last bits however near to 0 they are; 0 and 1 at infinite g.
__device__ __forceinline__ void gate_of(float g, float& z, float& keep) {
  const float s = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(g)), r = __builtin_amdgcn_rcpf(1.f + s);
  // the larger one as 1 - s r: the estimate's error counts s times, not once in every row that a state is kept for
  const float small = s * r, large = fmaf(-s, r, 1.f);
  z = g >= 0.f ? large : small;
  keep = g >= 0.f ? small : large;
}

__device__ __forceinline__ long bound_at(const void* p, int bytes, size_t s, long lo, long hi) {
  const long v = bytes == 8 ? ((const long*)p)[s] : (long)((const int*)p)[s];
  return v < lo ? lo : v > hi ? hi : v;
}

struct TileRows {
  int seq[TILE];                         // the sequence of a row, where it has one
  alignas(16) unsigned char flag[TILE];  // FIRST, LAST, VALID, ZERO
  int part[TPB / 64];
};

// Fills in the tile's rows.  Returns the sequences [s0, s1) that begin in the tile; those behind the last row belong to the last
// tile.  Sorted bounds give every row its sequence; unsorted ones give it some sequence, and no access leaves its array.
__device__ __forceinline__ void tile_rows(const ScanArgs& a, long t0, TileRows& t, size_t& s0, size_t& s1) {
  const long rows = (long)a.rows, t1 = t0 + TILE;
  const int i = threadIdx.x;
  const int none = a.zero_others ? ZERO : 0;
  if (!a.begin) {   // one sequence, or none at all
    if (i < TILE) {
      t.seq[i] = 0;
      t.flag[i] = t0 + i >= rows ? 0 : !a.n_seq ? none : VALID | (t0 + i == 0 ? FIRST : 0) | (t0 + i == rows - 1 ? LAST : 0);
    }
    s0 = 0;
    s1 = t0 == 0 && a.n_seq;
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
    int f = t0 + i < rows ? none : 0;
    if (s >= 0 && t0 + i < rows) {
      const long b = bound_at(a.begin, a.index_bytes, s, 0, rows), e = bound_at(a.end, a.index_bytes, s, b, rows), r = t0 + i;
      if (r >= b && r < e) f = VALID | (r == b ? FIRST : 0) | (r == e - 1 ? LAST : 0);
    }
    t.seq[i] = s;
    t.flag[i] = f;
  }
  __syncthreads();
}

// A thread's rows and features.  Features are independent, so a row's last lanes, where they would pass its end, take its last V
// features over again: they read, compute and write the same bits as the lanes that own them, and no access is cut short.  A
// feature's place in its workgroup (its slot) is its own all the same.  (Rows shorter than V: NARROW, element by element.)
template <class L>
struct Place {
  int grp, slot;
  size_t ch;   // its first feature
  int n;       // NARROW: features from there on
  __device__ Place(size_t c0, size_t hidden) {
    slot = threadIdx.x % L::LANES * L::V;
    grp = threadIdx.x / L::LANES;
    ch = c0 + slot;
    n = L::V;
    if (L::NARROW) {
      n = ch < hidden ? (int)(hidden - ch) : 0;
      if (!n) ch = 0;
    } else if (ch + L::V > hidden) {
      ch = hidden - L::V;
    }
  }
};

// The feature of a slot.
template <class L>
__device__ __forceinline__ size_t feature_of(int slot, size_t c0, size_t hidden) {
  const size_t ch = c0 + slot / L::V * L::V;
  return (!L::NARROW && ch + L::V > hidden ? hidden - L::V : ch) + slot % L::V;
}

// The groups of a tile's array: the tile's first row for all (in scalar registers), 32-bit offsets for the lanes.
template <class L, class E>
struct TileArray {
  E* base;
  unsigned off, step;
  __device__ TileArray(E* p, size_t stride, size_t tile, const Place<L>& at) {
    base = p + tile * TILE * stride;
    off = (unsigned)(at.grp * L::LS) * (unsigned)stride + (unsigned)at.ch;
    step = (unsigned)stride;
  }
  __device__ E* row(int i) const { return (E*)((char*)base + (off + i * step) * (unsigned)sizeof(E)); }
};

template <class L>
__device__ __forceinline__ void load_rows(const void* p, size_t stride, const Place<L>& at, size_t tile, int rows, Vec<typename L::E, L::V> (&v)[L::LS]) {
  const TileArray<L, const typename L::E> a((const typename L::E*)p, stride, tile, at);
#pragma unroll
  for (int i = 0; i < L::LS; ++i) {
    v[i].u = (typename Vec<typename L::E, L::V>::U)0u;
    if (at.grp * L::LS + i < rows) v[i] = load_group<L::V>(a.row(i), L::NARROW ? at.n : L::V);
  }
}

// A thread's features of a state, in 32 bits.
template <class L>
struct State {
  Vec<float> v[L::V / 4];
  __device__ float at(int k) const { return get(v[k / 4], k % 4); }
};
template <class L>
__device__ __forceinline__ State<L> load_state(const float* p, size_t row, const ScanArgs& a, const Place<L>& at) {
  State<L> s;
#pragma unroll
  for (int j = 0; j < L::V / 4; ++j) s.v[j] = load_vec(p + row * a.hidden + at.ch + 4 * j, L::NARROW ? at.n - 4 * j : 4);
  return s;
}
template <class L>
__device__ __forceinline__ void store_state(float* p, size_t row, const ScanArgs& a, const Place<L>& at, const float (&h)[L::V]) {
#pragma unroll
  for (int j = 0; j < L::V / 4; ++j) {
    const float o[4] = {h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]};
    store_vec(p + row * a.hidden + at.ch + 4 * j, pack<float>(o), L::NARROW ? at.n - 4 * j : 4);
  }
}

// A thread's flags, one byte a row; whether all rows of its wave are inner rows of a sequence.
template <class L>
struct Flags {
  unsigned w[L::LS / 4];
  bool plain;
  __device__ Flags(const TileRows& t, const Place<L>& at) {
    plain = true;
#pragma unroll
    for (int i = 0; i < L::LS / 4; ++i) {
      w[i] = ((const unsigned*)t.flag)[at.grp * (L::LS / 4) + i];
      plain = plain && w[i] == 0x01010101u * (unsigned)VALID;
    }
    plain = __all(plain);
  }
  __device__ int of(int i) const { return w[i / 4] >> (i % 4 * 8) & 0xff; }
};

// The states of a thread's rows with `flag` join what x holds: x + s, or x + keep s.  Four rows' loads are on their way together.
template <bool KEEP, class L>
__device__ __forceinline__ void take_in(const float* states, int flag, const ScanArgs& a, const TileRows& t, const Place<L>& at, const Flags<L>& f,
                                        const float (&keep)[L::LS][L::V], float (&x)[L::LS][L::V]) {
#pragma unroll
  for (int i0 = 0; i0 < L::LS; i0 += 4) {
    State<L> s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (f.of(i0 + i) & flag) s[i] = load_state<L>(states, t.seq[at.grp * L::LS + i0 + i], a, at);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (f.of(i0 + i) & flag)
#pragma unroll
        for (int k = 0; k < L::V; ++k) x[i0 + i][k] = KEEP ? fmaf(keep[i0 + i][k], s[i].at(k), x[i0 + i][k]) : x[i0 + i][k] + s[i].at(k);
  }
}

// The map of a thread's rows, from the first on.  With a cut among them it is a cut in every feature, whatever their gates hold.
template <bool PLAIN, class L>
__device__ __forceinline__ void map_forward(const Flags<L>& f, const float (&keep)[L::LS][L::V], const float (&zv)[L::LS][L::V], float (&p)[L::V],
                                            float (&q)[L::V]) {
  bool cuts = false;
#pragma unroll
  for (int k = 0; k < L::V; ++k) p[k] = 1.f, q[k] = 0.f;
#pragma unroll
  for (int i = 0; i < L::LS; ++i) {
    const bool cut = !PLAIN && (f.of(i) & (FIRST | VALID)) != VALID, none = !PLAIN && !(f.of(i) & VALID);
    cuts = cuts || cut;
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      const float qk = fmaf(keep[i][k], q[k], zv[i][k]);
      p[k] *= keep[i][k];
      q[k] = cut ? (none ? 0.f : zv[i][k]) : qk;
    }
  }
  if (!PLAIN)
#pragma unroll
    for (int k = 0; k < L::V; ++k) p[k] = cuts ? __uint_as_float(CUT) : p[k];
}

// The map of X over a thread's rows, from the last on.
template <bool PLAIN, class L>
__device__ __forceinline__ void map_back(const Flags<L>& f, const float (&keep)[L::LS][L::V], const float (&d)[L::LS][L::V], float (&p)[L::V],
                                         float (&q)[L::V]) {
  bool cuts = false;
#pragma unroll
  for (int k = 0; k < L::V; ++k) p[k] = 1.f, q[k] = 0.f;
#pragma unroll
  for (int i = L::LS - 1; i >= 0; --i) {
    const bool cut = !PLAIN && (f.of(i) & (FIRST | VALID)) != VALID;
    cuts = cuts || cut;
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      p[k] *= keep[i][k];
      q[k] = cut ? 0.f : keep[i][k] * (q[k] + d[i][k]);
    }
  }
  if (!PLAIN)
#pragma unroll
    for (int k = 0; k < L::V; ++k) p[k] = cuts ? __uint_as_float(CUT) : p[k];
}

// Per feature, the map of every thread's rows in front of its own (BACK: behind) inside the tile, and the tile's: through LDS, a
// part of the row groups and a feature to a lane.
template <class L>
struct __attribute__((aligned(16))) Maps {
  float p[L::TG][L::CH], q[L::TG][L::CH], tp[L::PARTS][L::CH], tq[L::PARTS][L::CH];
};
template <class L, bool BACK>
__device__ __forceinline__ void scan_groups(Maps<L>& m, const Place<L>& at, const float (&p)[L::V], const float (&q)[L::V]) {
#pragma unroll
  for (int k = 0; k < L::V; ++k) {
    m.p[at.grp][at.slot + k] = p[k];
    m.q[at.grp][at.slot + k] = q[k];
  }
  __syncthreads();
  constexpr int PER = L::TG / L::PARTS;
  const int part = threadIdx.x / L::CH, c = threadIdx.x % L::CH;
  float cp = 1.f, cq = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int g = part * PER + (BACK ? PER - 1 - i : i);
    const float gp = m.p[g][c], gq = m.q[g][c];
    m.p[g][c] = cp;
    m.q[g][c] = cq;
    compose(cp, cq, gp, gq);
  }
  m.tp[part][c] = cp;
  m.tq[part][c] = cq;
  __syncthreads();
}
// What comes into a thread's rows, from what comes into its part of the tile.
template <class L>
__device__ __forceinline__ float into_group(const Maps<L>& m, const Place<L>& at, int k, const float (&into)[L::PARTS][L::CH]) {
  const int c = at.slot + k;
  return apply(m.p[at.grp][c], m.q[at.grp][c], into[at.grp / (L::TG / L::PARTS)][c]);
}
// A slot to a lane: what comes into every part where x comes into the tile.
template <class L, bool BACK>
__device__ __forceinline__ void into_parts(const Maps<L>& m, int c, float x, float (&into)[L::PARTS][L::CH]) {
#pragma unroll
  for (int i = 0; i < L::PARTS; ++i) {
    const int w = BACK ? L::PARTS - 1 - i : i;
    into[w][c] = x;
    x = apply(m.tp[w][c], m.tq[w][c], x);
  }
}
template <class L, bool BACK>
__device__ __forceinline__ void tile_map(const Maps<L>& m, int c, float& p, float& q) {
  p = 1.f, q = 0.f;
#pragma unroll
  for (int i = 0; i < L::PARTS; ++i) compose(p, q, m.tp[BACK ? L::PARTS - 1 - i : i][c], m.tq[BACK ? L::PARTS - 1 - i : i][c]);
}

// ------------------------------------------------------------------ the hand-over between tiles
// Workspace: a ticket counter for every CH features, 64 bytes apart, then a word for every tile and slot and one for every group of
// tiles and slot, then the rows' flags and sequences, the same for all features.  Counters and words are EMPTY before the kernel; no map has
// those bits (a NaN is published as the one below).  The tiles of CH features are taken by ticket, in the order in which their states
// follow each other (the backward pass: from the last on): a workgroup waits only for tiles that running workgroups have taken, so
// every wait ends whatever else the GPU does.  (Another call that writes the same workspace at the same time, which amp.h forbids, could break
// that: a wait is given up after WAIT_TURNS looks, some seconds, so that the GPU is free again, and the states become NaN.  Looks are
// counted, not time, which goes by as well while the machine has the queue off the GPU.)
constexpr int GROUP = 4;   // tiles that share a word
constexpr int FAR = 16;    // groups in front that a wait looks at
constexpr int AHEAD = 4;   // words of them on their way together
constexpr unsigned EMPTY = 0xffffffffu, PUBLISHED_NAN = 0x7fc00000u;
constexpr int WAIT_TURNS = 1 << 22;

__device__ __forceinline__ unsigned long long word_of(float p, float q) {
  unsigned a = __float_as_uint(p), b = __float_as_uint(q);
  a = a == EMPTY ? PUBLISHED_NAN : a;
  b = b == EMPTY ? PUBLISHED_NAN : b;
  return (unsigned long long)b << 32 | a;
}
__device__ __forceinline__ float word_p(unsigned long long w) { return __uint_as_float((unsigned)w); }
__device__ __forceinline__ float word_q(unsigned long long w) { return __uint_as_float((unsigned)(w >> 32)); }
__device__ __forceinline__ bool word_there(unsigned long long w) { return (unsigned)w != EMPTY && (unsigned)(w >> 32) != EMPTY; }
__device__ __forceinline__ bool word_cut(unsigned long long w) { return (unsigned)w == CUT; }

struct Hand {
  unsigned* tickets;
  unsigned long long *words, *groups;
  int* seq;
  unsigned char* flag;
  size_t tiles, slots;   // slots: the features in whole workgroups
  __host__ __device__ static size_t slots_of(size_t hidden) { return (hidden + 63) / 64 * 64; }
  // a ticket counter for every 64 slots, words for all slots
  __host__ __device__ static size_t clear_bytes(size_t tiles, size_t hidden) { return slots_of(hidden) * (1 + (tiles + tiles / GROUP) * 8); }
  __device__ Hand(const ScanArgs& a, size_t tiles_) : tiles(tiles_), slots(slots_of(a.hidden)) {
    tickets = (unsigned*)a.workspace;
    words = (unsigned long long*)((char*)a.workspace + slots);
    groups = words + tiles * slots;
    seq = (int*)((char*)a.workspace + clear_bytes(tiles, a.hidden));
    flag = (unsigned char*)(seq + tiles * TILE);
  }
  __device__ unsigned long long load(const unsigned long long* of, size_t i, size_t slot) const {
    return __hip_atomic_load(of + i * slots + slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ void store(unsigned long long* of, size_t i, size_t slot, float p, float q) const {
    __hip_atomic_store(of + i * slots + slot, word_of(p, q), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
};

// One wave, a slot to a lane: publishes the tile's map and returns what comes into the tile: what comes into its group of GROUP tiles,
// through the maps of the group's tiles in front.  A group's last tile publishes the group's map, and once what comes into the group is
// known the map that gives what goes out.  A wait for that looks at the word of the group in front, which is mostly what it needs, and
// at one word of each of FAR groups: where the state behind the nearest is not known yet, it is formed from the nearest known one over
// the maps between, up to AHEAD words on their way together.
// A chain of states over single tiles costs 0.17 us a tile, and that is the time of a call with few features, whose tiles all run at
// once; in groups it is 0.07 (one sequence of 524,288 x 256 bf16: 709 and 285 us; 131,072 x 640: 209 and 141; 65,536 x 2,048: 198 and
// 185).  The group's words cost 2 to 4 % where no chain is waited for (the backward pass of 65,536 x 2,048: 324 and 332 us).
__device__ __forceinline__ float hand_over(const Hand& h, size_t order, size_t slot0, float p, float q) {
  const int lane = threadIdx.x & 63, r = (int)(order % GROUP);
  const size_t slot = slot0 + lane, g = order / GROUP, first = order - r;
  const bool closes = r == GROUP - 1;
  const int far = g < FAR ? (int)g : FAR;
  if (!closes) h.store(h.words, order, slot, p, q);
  float lp = 1.f, lq = 0.f, gp = p, gq = q, x = 0.f;   // the maps of the group's tiles in front, and with this one; what comes into the group
  bool local = r == 0, known = g == 0;
  for (int turn = 0;; ++turn) {
    unsigned long long w[GROUP - 1], next = 0, s = ~0ull;
    if (!local)
#pragma unroll
      for (int i = 0; i < GROUP - 1; ++i)
        if (i < r) w[i] = h.load(h.words, first + i, slot);
    if (!known) {
      next = h.load(h.groups, g - 1, slot);
      if (lane < far) s = h.load(h.groups, g - 1 - lane, slot0);
    }
    if (!local) {
      bool all = true;
      lp = 1.f, lq = 0.f;
#pragma unroll
      for (int i = 0; i < GROUP - 1; ++i)
        if (i < r) {
          all = all && word_there(w[i]);
          compose(lp, lq, word_p(w[i]), word_q(w[i]));
        }
      local = __all(all);
      if (local) {
        gp = lp, gq = lq;
        compose(gp, gq, p, q);
        if (closes) h.store(h.groups, g, slot, gp, gq);
      }
    }
    // a sequence begins in the group's tiles in front (gp is a cut in every lane with lp: what goes out of the group is published)
    if (local && __all(is_cut(lp))) return lq;
    if (!known) {
      const unsigned long long cuts = __ballot(word_there(s) && word_cut(s)), there = __ballot(word_there(s));
      int n = cuts ? __ffsll(cuts) : 0;   // groups to go back to
      if (n && (~there & ~0ull >> (64 - n))) n = 0;   // (one between is missing)
      if (__all(word_there(next) && word_cut(next))) n = 1;
      if (n) {
        bool all = true;
        x = 0.f;
        for (int at = n; at > 0; at -= AHEAD) {   // from the farthest on, up to AHEAD words on their way together
          unsigned long long v[AHEAD];
#pragma unroll
          for (int i = 0; i < AHEAD; ++i)
            if (at - i > 1) v[i] = h.load(h.groups, g - (at - i), slot);
#pragma unroll
          for (int i = 0; i < AHEAD; ++i)
            if (at - i > 0) {
              const unsigned long long u = at - i > 1 ? v[i] : next;
              all = all && word_there(u) && (at - i < n || word_cut(u));
              x = apply(word_p(u), word_q(u), x);
            }
        }
        known = __all(all);
      }
    }
    if (local && known) {
      // a group that cuts the states itself has published what goes out already
      if (closes && !__all(is_cut(gp))) h.store(h.groups, g, slot, __uint_as_float(CUT), apply(gp, gq, x));
      return apply(lp, lq, x);
    }
    if (turn == WAIT_TURNS) {
      if (closes) h.store(h.groups, g, slot, __uint_as_float(CUT), __uint_as_float(PUBLISHED_NAN));
      return __uint_as_float(PUBLISHED_NAN);
    }
    __builtin_amdgcn_s_sleep(2);
  }
}

// The 64 features of this workgroup: `blocks` consecutive workgroups have one each, every time shifted by one.  Workgroups go to the
// eight dies in turn; were the features not shifted, a die would read the same few columns of every row, and with them few of its
// L2's channels (65,536 x 2,048 bf16, forward: 255 us without the shift, 230 with it).
__device__ __forceinline__ size_t feature_block(size_t blocks) { return (blockIdx.x % blocks + blockIdx.x / blocks) % blocks; }

// Its place in the order of its features' tiles.
__device__ __forceinline__ size_t take_ticket(const Hand& h, size_t block, unsigned* shared) {
  if (h.tiles == 1) return 0;
  if (threadIdx.x == 0)   // the counters start at -1
    *shared = __hip_atomic_fetch_add(h.tickets + block * 16, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
  __syncthreads();
  return *shared;
}

// Sequences without rows hand their state through.
__device__ __forceinline__ void pass_through(const ScanArgs& a, size_t s0, size_t s1, float* out, const float* from) {
  for (size_t s = s0; s < s1; ++s) {
    const long b = a.begin ? bound_at(a.begin, a.index_bytes, s, 0, (long)a.rows) : 0;
    const long e = a.begin ? bound_at(a.end, a.index_bytes, s, b, (long)a.rows) : (long)a.rows;
    if (e <= b)
      for (size_t ch = threadIdx.x; ch < a.hidden; ch += blockDim.x) out[s * a.hidden + ch] = from ? from[s * a.hidden + ch] : 0.f;
  }
}

// In front of the scan over several tiles: the rows' flags and sequences (a tile to a workgroup), and the words EMPTY.
template <bool BACK>
__global__ __launch_bounds__(TPB) void scan_plan_kernel(ScanArgs a, size_t tiles) {
  __shared__ TileRows t;
  const Hand hand(a, tiles);
  v4u* w = (v4u*)a.workspace;
  const size_t n16 = Hand::clear_bytes(tiles, a.hidden) / 16;
  for (size_t i = (size_t)blockIdx.x * TPB + threadIdx.x; i < n16; i += (size_t)gridDim.x * TPB) w[i] = (v4u){EMPTY, EMPTY, EMPTY, EMPTY};
  for (size_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    size_t s0, s1;
    tile_rows(a, (long)tile * TILE, t, s0, s1);
    const int i = threadIdx.x;
    if (i < TILE) {
      hand.seq[tile * TILE + i] = t.seq[i];
      hand.flag[tile * TILE + i] = t.flag[i];
    }
    float* out = BACK ? a.dh0 : a.last;
    if (out) pass_through(a, s0, s1, out, BACK ? a.dlast : a.h0);
    __syncthreads();
  }
}

__device__ __forceinline__ int rows_of(const ScanArgs& a, size_t tile) {
  const size_t left = a.rows - tile * TILE;
  return left < TILE ? (int)left : TILE;
}

// The rows' flags and sequences of a tile: planned (several tiles), fetched in front of the tile itself and there when it is; or found
// here.
struct RowsAhead {
  int seq;
  unsigned flag;
  __device__ RowsAhead(const Hand& hand, size_t tile) {
    if (hand.tiles > 1) {
      if (threadIdx.x < TILE) seq = hand.seq[tile * TILE + threadIdx.x];
      if (threadIdx.x < TILE / 4) flag = ((const unsigned*)hand.flag)[tile * (TILE / 4) + threadIdx.x];
    }
  }
  __device__ void put(const ScanArgs& a, const Hand& hand, TileRows& t, float* out, const float* from) const {
    if (hand.tiles > 1) {
      if (threadIdx.x < TILE) t.seq[threadIdx.x] = seq;
      if (threadIdx.x < TILE / 4) ((unsigned*)t.flag)[threadIdx.x] = flag;
    } else {
      size_t s0, s1;
      tile_rows(a, 0, t, s0, s1);
      if (blockIdx.x == 0 && out) pass_through(a, s0, s1, out, from);
    }
  }
};

template <bool PLAIN, class L>
__device__ __forceinline__ void write_forward(const ScanArgs& a, const TileRows& t, const Place<L>& at, size_t tile, const Flags<L>& f,
                                              const float (&keep)[L::LS][L::V], const float (&zv)[L::LS][L::V], float (&h)[L::V]) {
  typedef typename L::E T;
  const TileArray<L, T> out((T*)a.h, a.h_stride, tile, at);
#pragma unroll
  for (int i = 0; i < L::LS; ++i) {
    const bool first = !PLAIN && (f.of(i) & FIRST);
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      const float next = fmaf(keep[i][k], h[k], zv[i][k]);
      h[k] = first ? zv[i][k] : next;
    }
    if (a.h && (PLAIN || (f.of(i) & (VALID | ZERO)))) {
      Vec<T, L::V> o = pack<T>(h);
      if (!PLAIN && (f.of(i) & ZERO)) o = {};
      store_vec(out.row(i), o, L::NARROW ? at.n : L::V);
    }
    if (!PLAIN && (f.of(i) & LAST) && a.last) store_state<L>(a.last, t.seq[at.grp * L::LS + i], a, at, h);
  }
}

template <class L, bool TANH>
__global__ __launch_bounds__(TPB, 4) void scan_forward_kernel(ScanArgs a, size_t tiles) {
  __shared__ TileRows t;
  __shared__ Maps<L> m;
  __shared__ __attribute__((aligned(16))) float into[L::PARTS][L::CH];
  __shared__ unsigned ticket;
  const Hand hand(a, tiles);
  const size_t blocks = (a.hidden + L::CH - 1) / L::CH, block = feature_block(blocks), c0 = block * L::CH;
  const Place<L> at(c0, a.hidden);
  const size_t order = take_ticket(hand, block, &ticket);
  const RowsAhead ahead(hand, order);
  Vec<typename L::E, L::V> g[L::LS], c[L::LS];
  load_rows<L>(a.gate, a.gate_stride, at, order, rows_of(a, order), g);
  load_rows<L>(a.cand, a.cand_stride, at, order, rows_of(a, order), c);
  ahead.put(a, hand, t, a.last, a.h0);
  float keep[L::LS][L::V], zv[L::LS][L::V];
#pragma unroll
  for (int i = 0; i < L::LS; ++i)
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      float z;
      gate_of(get(g[i], k), z, keep[i][k]);
      zv[i][k] = z * (TANH ? tanh_(get(c[i], k)) : get(c[i], k));
    }
  __syncthreads();
  const Flags<L> f(t, at);
  float p[L::V], q[L::V];
  if (f.plain) {
    map_forward<true, L>(f, keep, zv, p, q);
  } else {
    if (a.h0) take_in<true, L>(a.h0, FIRST, a, t, at, f, keep, zv);
    map_forward<false, L>(f, keep, zv, p, q);
  }
  scan_groups<L, false>(m, at, p, q);
  if (threadIdx.x < L::CH) {
    float x = 0.f;
    if (tiles > 1) {
      float tp, tq;
      tile_map<L, false>(m, threadIdx.x, tp, tq);
      x = hand_over(hand, order, c0, tp, tq);
    }
    into_parts<L, false>(m, threadIdx.x, x, into);
  }
  __syncthreads();
  float h[L::V];
#pragma unroll
  for (int k = 0; k < L::V; ++k) h[k] = into_group<L>(m, at, k, into);
  if (a.carry && at.grp == 0) store_state<L>(a.carry, order, a, at, h);
  if (f.plain)
    write_forward<true, L>(a, t, at, order, f, keep, zv, h);
  else
    write_forward<false, L>(a, t, at, order, f, keep, zv, h);
}

// Backward: X_t = keep_t G_t is what a row hands to the row in front of it, G_t = d_t + X_{t+1}, d_t = dh_t (+ dlast at a last
// row); a first row hands it to dh0 and nothing to the row in front, so the cuts are the forward pass's.  h_{t-1} is formed again
// from the carry in 32 bits: a row less to read than with h, and none of its rounding.
template <bool PLAIN, class L>
__device__ __forceinline__ void states_before(const Flags<L>& f, const float (&keep)[L::LS][L::V], float (&x)[L::V], float (&h)[L::LS][L::V]) {
#pragma unroll
  for (int i = 0; i < L::LS; ++i)   // h holds z v, and behind this the state in front of the row (at a first row the next pass puts h0)
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      const float zv = h[i][k], next = fmaf(keep[i][k], x[k], zv);
      h[i][k] = x[k];
      x[k] = !PLAIN && (f.of(i) & FIRST) ? zv : next;
    }
}

template <bool PLAIN, class L, bool TANH>
__device__ __forceinline__ void write_back(const ScanArgs& a, const TileRows& t, const Place<L>& at, size_t tile, const Flags<L>& f,
                                           const float (&keep)[L::LS][L::V], const float (&z)[L::LS][L::V], const float (&v)[L::LS][L::V],
                                           const float (&h)[L::LS][L::V], const float (&d)[L::LS][L::V], float (&x)[L::V]) {
  typedef typename L::E T;
  const TileArray<L, T> out_g((T*)a.dgate, a.dgate_stride, tile, at), out_c((T*)a.dcand, a.dcand_stride, tile, at);
#pragma unroll
  for (int i = L::LS - 1; i >= 0; --i) {
    float og[L::V], oc[L::V];
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      const float G = d[i][k] + x[k], zG = z[i][k] * G;
      x[k] = keep[i][k] * G;
      og[k] = zG * keep[i][k] * (v[i][k] - h[i][k]);
      oc[k] = TANH ? zG * fmaf(-v[i][k], v[i][k], 1.f) : zG;
    }
    if (PLAIN || (f.of(i) & (VALID | ZERO))) {
      Vec<T, L::V> vg = pack<T>(og), vc = pack<T>(oc);
      if (!PLAIN && (f.of(i) & ZERO)) vg = vc = {};
      store_vec(out_g.row(i), vg, L::NARROW ? at.n : L::V);
      store_vec(out_c.row(i), vc, L::NARROW ? at.n : L::V);
    }
    if (!PLAIN && (f.of(i) & FIRST) && a.dh0) store_state<L>(a.dh0, t.seq[at.grp * L::LS + i], a, at, x);
    if (!PLAIN)
#pragma unroll
      for (int k = 0; k < L::V; ++k) x[k] = (f.of(i) & (FIRST | VALID)) != VALID ? 0.f : x[k];
  }
}

template <class L, bool TANH>
__global__ __launch_bounds__(TPB, 2) void scan_backward_kernel(ScanArgs a, size_t tiles) {
  __shared__ TileRows t;
  __shared__ Maps<L> m, back;
  __shared__ __attribute__((aligned(16))) float into[L::PARTS][L::CH], before[L::PARTS][L::CH];
  __shared__ unsigned ticket;
  const Hand hand(a, tiles);
  const size_t blocks = (a.hidden + L::CH - 1) / L::CH, block = feature_block(blocks), c0 = block * L::CH;
  const Place<L> at(c0, a.hidden);
  const size_t order = take_ticket(hand, block, &ticket), tile = tiles - 1 - order;
  const RowsAhead ahead(hand, tile);
  Vec<typename L::E, L::V> g[L::LS], c[L::LS], dh[L::LS];
  load_rows<L>(a.gate, a.gate_stride, at, tile, rows_of(a, tile), g);
  load_rows<L>(a.dh, a.dh_stride, at, tile, rows_of(a, tile), dh);
  load_rows<L>(a.cand, a.cand_stride, at, tile, rows_of(a, tile), c);
  ahead.put(a, hand, t, a.dh0, a.dlast);
  float keep[L::LS][L::V], z[L::LS][L::V], v[L::LS][L::V], d[L::LS][L::V], h[L::LS][L::V];
#pragma unroll
  for (int i = 0; i < L::LS; ++i) {
#pragma unroll
    for (int k = 0; k < L::V; ++k) {
      gate_of(get(g[i], k), z[i][k], keep[i][k]);
      d[i][k] = get(dh[i], k);
      v[i][k] = TANH ? tanh_(get(c[i], k)) : get(c[i], k);
      h[i][k] = z[i][k] * v[i][k];
    }
    // a row's tangents are formed here: moved behind the barrier, all of them side by side do not fit the registers
    if (TANH)
#pragma unroll
      for (int k = 0; k < L::V; ++k) asm volatile("" : "+v"(v[i][k]));
  }
  __syncthreads();
  const Flags<L> f(t, at);
  float p[L::V], q[L::V], x[L::V];
  if (f.plain) {
    map_back<true, L>(f, keep, d, p, q);
  } else {
    if (a.dlast) take_in<false, L>(a.dlast, LAST, a, t, at, f, keep, d);
    map_back<false, L>(f, keep, d, p, q);
  }
  scan_groups<L, true>(back, at, p, q);
  if (f.plain) {
    map_forward<true, L>(f, keep, h, p, q);
  } else {
    if (a.h0) take_in<true, L>(a.h0, FIRST, a, t, at, f, keep, h);
    map_forward<false, L>(f, keep, h, p, q);
  }
  scan_groups<L, false>(m, at, p, q);
  if (threadIdx.x < L::CH) {
    float in = 0.f;
    if (tiles > 1) {
      float tp, tq;
      tile_map<L, true>(back, threadIdx.x, tp, tq);
      in = hand_over(hand, order, c0, tp, tq);
    }
    into_parts<L, true>(back, threadIdx.x, in, into);
  } else if (threadIdx.x < 2 * L::CH) {   // beside it
    const int s = threadIdx.x - L::CH;
    const bool in = !L::NARROW || (size_t)s < a.hidden;
    into_parts<L, false>(m, s, in ? a.carry_in[tile * a.hidden + feature_of<L>(s, c0, a.hidden)] : 0.f, before);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < L::V; ++k) x[k] = into_group<L>(m, at, k, before);
  if (f.plain) {
    states_before<true, L>(f, keep, x, h);
  } else {
    states_before<false, L>(f, keep, x, h);
#pragma unroll
    for (int i = 0; i < L::LS; ++i)
      if (f.of(i) & FIRST)
#pragma unroll
        for (int k = 0; k < L::V; ++k) h[i][k] = 0.f;
    if (a.h0) take_in<false, L>(a.h0, FIRST, a, t, at, f, keep, h);
  }
#pragma unroll
  for (int k = 0; k < L::V; ++k) x[k] = into_group<L>(back, at, k, into);
  if (f.plain)
    write_back<true, L, TANH>(a, t, at, tile, f, keep, z, v, h, d, x);
  else
    write_back<false, L, TANH>(a, t, at, tile, f, keep, z, v, h, d, x);
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
size_t bytes_of(size_t tiles, size_t hidden) {
  return tiles == 1 ? 0 : (Hand::clear_bytes(tiles, hidden) + tiles * TILE * 5 + 15) / 16 * 16;
}

template <class L, bool BACK>
hipError_t run(void (*kernel)(ScanArgs, size_t), const ScanArgs& a, hipStream_t stream) {
  const size_t tiles = tiles_of(a.rows), blocks = (a.hidden + L::CH - 1) / L::CH;
  if (tiles > 1) {
    const hipError_t e = launch(scan_plan_kernel<BACK>, dim3((unsigned)(tiles < 1024 ? tiles : 1024)), dim3(TPB), 0, stream, a, tiles);
    if (e != hipSuccess) return e;
  }
  return launch(kernel, dim3((unsigned)(blocks * tiles)), dim3(TPB), 0, stream, a, tiles);
}

}  // namespace

extern "C" size_t amp_scan_carry_rows(int, size_t rows, size_t) { return tiles_of(rows); }
extern "C" size_t amp_scan_workspace_bytes(int, size_t rows, size_t hidden) { return bytes_of(tiles_of(rows), hidden); }

namespace {
template <class T, bool NARROW>
hipError_t forward(int tanh, const ScanArgs* a, hipStream_t stream) {
  typedef Lay<T, NARROW> L;
  return run<L, false>(tanh ? scan_forward_kernel<L, true> : scan_forward_kernel<L, false>, *a, stream);
}
template <class T, bool NARROW>
hipError_t backward(int tanh, const ScanArgs* a, hipStream_t stream) {
  typedef Lay<T, NARROW> L;
  return run<L, true>(tanh ? scan_backward_kernel<L, true> : scan_backward_kernel<L, false>, *a, stream);
}

}  // namespace

extern "C" hipError_t amp_scan_forward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream) {
  OPS_BY_TYPE(dtype, return a->hidden < Lay<T, false>::V ? forward<T, true>(tanh, a, stream) : forward<T, false>(tanh, a, stream));
}

extern "C" hipError_t amp_scan_backward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream) {
  OPS_BY_TYPE(dtype, return a->hidden < Lay<T, false>::V ? backward<T, true>(tanh, a, stream) : backward<T, false>(tanh, a, stream));
}

extern "C" hipError_t amp_scan_step_launch(int dtype, int tanh, const ScanStepArgs* a, hipStream_t stream) {
  const size_t v = dtype == 0 ? 4 : 8, blocks = (a->rows * ((a->hidden + v - 1) / v) + TPB - 1) / TPB;
  const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
  OPS_BY_TYPE(dtype, return tanh ? launch(scan_step_kernel<T, true>, grid, dim3(TPB), 0, stream, *a)
                                 : launch(scan_step_kernel<T, false>, grid, dim3(TPB), 0, stream, *a));
}
