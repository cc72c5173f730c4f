"""The gated recurrence's maps and the hand-over of states between its tiles, taken from their source and compiled for the host: the 64
lanes of a wave take turns from one meeting (ballot, vote) to the next.  Where tiles run one after the other in the order of their tickets,
everything a tile asks for is there when it asks: no wait may take a second turn, whatever the rows hold."""
import ctypes as ct
import os
import re
import subprocess

import numpy as np
import pytest

from paper_1705_09786_amd import build

HOST = r"""
#include <stddef.h>
#include <stdint.h>
#include <string.h>
#include <ucontext.h>
#include <algorithm>
#include <cmath>
#include <vector>
#define __device__
#define __host__
#define __forceinline__ inline
static float __uint_as_float(unsigned u) { float f; memcpy(&f, &u, 4); return f; }
static unsigned __float_as_uint(float f) { unsigned u; memcpy(&u, &f, 4); return u; }
struct ScanArgs { size_t hidden; void* workspace; };

// ---- a wave: every lane runs up to the next meeting, then all of them go on with its result
struct Wave {
  ucontext_t lane[64];
  unsigned long long vote, result;
  int turns;
  size_t order;
  float p[64], q[64], in[64];
  bool done[64];
};
static ucontext_t g_main;
static Wave* g_wave;
static int g_at;
static long g_clock;
static struct { unsigned x; } threadIdx;
static unsigned long long ballot(bool v) {
  if (v) g_wave->vote |= 1ull << g_at;
  swapcontext(&g_wave->lane[g_at], &g_main);
  return g_wave->result;
}
#define __ballot(v) ballot(v)
#define __all(v) (ballot(v) == ~0ull)
#define __ffsll(v) __builtin_ffsll((long long)(v))
#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_load(p, order, scope) (*(p))
#define __hip_atomic_store(p, v, order, scope) (*(p) = (v))
static long wall_clock64() { return g_clock; }
#define __builtin_amdgcn_s_sleep(n) (g_wave->turns += g_at == 63)
constexpr int TILE = 128;
%s

// ---- the maps of a thread's rows: its flags, and four features
struct Lay { static constexpr int LS = 8, V = 4; };
template <class L>
struct Flags {
  const unsigned char* f;
  int of(int i) const { return f[i]; }
};
%s

// ---- the waves of several tiles, a turn each
static const Hand* g_hand;
static void lane_main() {
  Wave& w = *g_wave;
  const int lane = g_at;
  w.in[lane] = hand_over(*g_hand, w.order, 0, w.p[lane], w.q[lane]);
  w.done[lane] = true;
}
constexpr size_t STACK = 32768;
static void start(Wave& w, char* stacks) {
  w.vote = w.result = 0;
  w.turns = 0;
  for (int l = 0; l < 64; ++l) {
    w.done[l] = false;
    getcontext(&w.lane[l]);
    w.lane[l].uc_stack.ss_sp = stacks + l * STACK;
    w.lane[l].uc_stack.ss_size = STACK;
    w.lane[l].uc_link = &g_main;
    makecontext(&w.lane[l], lane_main, 0);
  }
}
// On to the wave's next meeting: 1 = all lanes are done, 0 = none, -1 = they parted.
static int step(Wave& w) {
  g_wave = &w;
  w.vote = 0;
  for (int l = 0; l < 64; ++l) {
    g_at = l;
    threadIdx.x = l;
    swapcontext(&g_main, &w.lane[l]);
  }
  w.result = w.vote;
  const int n = std::count(w.done, w.done + 64, true);
  return n == 64 ? 1 : n ? -1 : 0;
}

// rows x 64 keeps, terms and flags (tiles * 128 rows from the first on; back = 1: the states run from the last on) -> what comes into
// every tile, and the extra turns of its wait.  Up to `together` tiles are under way, the later ones first in every round of turns;
// `jump` ticks of the clock go by between two rounds.
extern "C" int run(int tiles, int back, int together, long jump, const float* keep, const float* term, const unsigned char* flag, float* in,
                   int* turns) {
  std::vector<char> ws(Hand::clear_bytes(tiles, 64) + 64 + tiles * 5 * TILE);
  memset(ws.data(), 0xff, ws.size());
  ScanArgs a = {64, ws.data()};
  const Hand hand(a, tiles);
  g_hand = &hand;
  g_clock = 0;
  static std::vector<char> stacks;
  stacks.resize(std::max(stacks.size(), together * 64 * STACK));
  std::vector<Wave> waves(tiles);
  for (int order = 0; order < tiles; ++order) {
    const int tile = back ? tiles - 1 - order : order;
    Wave& w = waves[order];
    w.order = order;
    for (int c = 0; c < 64; c += 4) {
      float tp[4] = {1, 1, 1, 1}, tq[4] = {0, 0, 0, 0};
      for (int g = 0; g < TILE / 8; ++g) {
        const int r0 = tile * TILE + (back ? TILE / 8 - 1 - g : g) * 8;
        float k[8][4], t[8][4], gp[4], gq[4];
        for (int i = 0; i < 8; ++i)
          for (int j = 0; j < 4; ++j) k[i][j] = keep[(r0 + i) * 64 + c + j], t[i][j] = term[(r0 + i) * 64 + c + j];
        const Flags<Lay> f = {flag + r0};
        if (back)
          map_back<false, Lay>(f, k, t, gp, gq);
        else
          map_forward<false, Lay>(f, k, t, gp, gq);
        for (int j = 0; j < 4; ++j) compose(tp[j], tq[j], gp[j], gq[j]);
      }
      for (int j = 0; j < 4; ++j) w.p[c + j] = tp[j], w.q[c + j] = tq[j];
    }
  }
  for (int first = 0; first < tiles; first += together) {
    const int end = std::min(tiles, first + together);
    std::vector<int> state(end - first, 0);
    for (int t = first; t < end; ++t) start(waves[t], stacks.data() + (t - first) * 64 * STACK);
    for (int round = 0; std::count(state.begin(), state.end(), 1) < end - first; ++round) {
      for (int t = end - 1; t >= first; --t)
        if (!state[t - first] && (state[t - first] = step(waves[t])) < 0) return -1;
      g_clock += jump;
      if (round > 100000) return -2;
    }
  }
  for (int t = 0; t < tiles; ++t) memcpy(in + t * 64, waves[t].in, sizeof waves[t].in), turns[t] = waves[t].turns;
  return 0;
}
"""


def section(text, begin, end):
    return text[text.index(begin):text.index(end, text.index(begin))]


@pytest.fixture(scope="module")
def hand_over(tmp_path_factory):
    text = open(os.path.join(build.HERE, "csrc", "amp_scan.hip")).read()
    maps = section(text, "constexpr unsigned CUT", "// z = 1 / (1 + e^-g)")
    words = section(text, "constexpr int GROUP", "// The 64 features of this workgroup")
    rows = section(text, "// The map of a thread's rows, from the first on", "// Per feature, the map of every thread's rows in front")
    tmp = tmp_path_factory.mktemp("hand")
    src, so = tmp / "h.cpp", tmp / "h.so"
    src.write_text(HOST % (maps + words.replace("#pragma unroll", ""), rows.replace("#pragma unroll", "")))
    p = subprocess.run(["g++", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-std=c++17", str(src), "-o", str(so)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout
    lib = ct.CDLL(str(so))

    def call(keep, term, flag, back, together=1, jump=0):
        tiles = keep.shape[0] // 128
        into, turns = np.zeros((tiles, 64), np.float32), np.zeros(tiles, np.int32)
        ptr = lambda a, t: np.ascontiguousarray(a).ctypes.data_as(ct.POINTER(t))
        keep, term, flag = np.ascontiguousarray(keep), np.ascontiguousarray(term), np.ascontiguousarray(flag)
        assert lib.run(tiles, int(back), together, ct.c_long(jump), ptr(keep, ct.c_float), ptr(term, ct.c_float), ptr(flag, ct.c_uint8),
                       ptr(into, ct.c_float), ptr(turns, ct.c_int)) == 0
        return into, turns
    return call


FIRST, LAST, VALID = 1, 2, 4
TILES = 11   # two whole groups of tiles and most of a third


def rows_of(begins, rows, seed=0):
    """Keeps, terms and flags of sequences that begin at `begins`, one behind the other."""
    rng = np.random.default_rng(seed)
    keep = rng.uniform(0.6, 1.0, (rows, 64)).astype(np.float32)
    term = rng.standard_normal((rows, 64)).astype(np.float32)
    flag = np.full(rows, VALID, np.uint8)
    for b in begins:
        flag[b] |= FIRST
        if b:
            flag[b - 1] |= LAST
    flag[rows - 1] |= LAST
    return keep, term, flag


def serial(keep, term, flag, back):
    """What comes into every tile, in 64 bits, in the order of the tiles' tickets."""
    k, t, x, out = keep.astype(np.float64), term.astype(np.float64), np.zeros(64), []
    rows = keep.shape[0]
    for n, r in enumerate(range(rows - 1, -1, -1) if back else range(rows)):
        if n % 128 == 0:
            out.append(x)
        if back:
            x = np.zeros(64) if flag[r] & FIRST else k[r] * (t[r] + x)
        else:
            x = t[r] if flag[r] & FIRST else k[r] * x + t[r]
    return np.stack(out)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("begins", [[0], [0, 700], [0, 5, 130, 390, 391, 900], list(range(0, TILES * 128, 128))])
def test_states_are_the_serial_ones(hand_over, begins, back):
    keep, term, flag = rows_of(begins, TILES * 128)
    into, turns = hand_over(keep, term, flag, back)
    want = serial(keep, term, flag, back)
    assert not turns.any()
    # keeps of at most 1 and some 0.8 in the mean: a state is a sum of terms of size 4 at most over some 10 rows, each with the rounding
    # of its row and of up to 40 maps behind it
    assert np.abs(into - want).max() <= 2.0 ** -24 * 4 * 10 * 50


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("begins", [[0], [0, 700], [0, 5, 130, 390, 391, 900]])
@pytest.mark.parametrize("together", [2, 3, 4, 5, TILES])
def test_states_do_not_depend_on_who_comes_first(hand_over, begins, back, together):
    """Tiles under way at once, the later ones ahead of those that they wait for: the same bits.  Also where minutes go by meanwhile, as
    they do for a process whose queue the machine takes off the GPU: a wait is not given up for that."""
    keep, term, flag = rows_of(begins, TILES * 128, seed=together)
    want, _ = hand_over(keep, term, flag, back)
    for jump in (0, 60 * 100000000):
        got, turns = hand_over(keep, term, flag, back, together, jump)
        assert (got.view(np.int32) == want.view(np.int32)).all() and turns.max() > 0


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("slot", [0, 5, 63, None])
@pytest.mark.parametrize("begins", [[0], [0, 300], [0, 200, 640, 1153], list(range(0, TILES * 128, 64))])
def test_a_gate_that_is_no_number_stays_in_its_feature_and_sequence(hand_over, begins, slot, back):
    rows = TILES * 128
    keep, term, flag = rows_of(begins, rows)
    want, _ = hand_over(keep, term, flag, back)
    for tile in range(TILES):
        for r in (tile * 128, tile * 128 + 3, tile * 128 + 70, tile * 128 + 127):
            k, t = keep.copy(), term.copy()
            k[r, slot if slot is not None else slice(None)] = np.nan
            if not back:
                t[r, slot if slot is not None else slice(None)] = np.nan
            got, turns = hand_over(k, t, flag, back)
            assert not turns.any(), (r, turns)
            bad = np.isnan(serial(k, t, flag, back))
            assert (np.isnan(got) == bad).all(), (r, np.argwhere(np.isnan(got) != bad)[:3])
            assert (got.view(np.int32)[~bad] == want.view(np.int32)[~bad]).all(), r
