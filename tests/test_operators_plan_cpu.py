"""How the gated delta rule divides its rows, taken from its source and compiled for the host: the workspace's parts, the plan kernel (its
threads take turns from one meeting, a shuffle or a barrier, to the next), and what every workgroup finds for itself from those."""
import ctypes as ct
import os
import subprocess

import numpy as np
import pytest

from paper_1705_09786_amd import build

HOST = r"""
#include <stddef.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>
#include <vector>
#define __device__
#define __host__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(n)
#define __shared__ static
struct dim3 { unsigned x, y; dim3(unsigned x_ = 1, unsigned y_ = 1) : x(x_), y(y_) {} };
typedef int hipError_t;
typedef void* hipStream_t;
constexpr int hipSuccess = 0;
static long max(long a, long b) { return a > b ? a : b; }
static struct { unsigned x; } threadIdx;
%s

// ---- a workgroup: every thread runs up to the next meeting, then all of them go on
static ucontext_t g_main, g_thread[1024];
static long g_slot[2][1024];
static int g_parity[1024], g_left;
static void meet() {
  const unsigned me = threadIdx.x;
  swapcontext(&g_thread[me], &g_main);
  threadIdx.x = me;
}
static void __syncthreads() { meet(); }
static long exchange(long v, unsigned from) {
  const int p = g_parity[threadIdx.x];
  g_parity[threadIdx.x] ^= 1;
  g_slot[p][threadIdx.x] = v;
  meet();
  return g_slot[p][from];
}
static long __shfl_up(long v, int d, int) { return exchange(v, (int)(threadIdx.x & 63) >= d ? threadIdx.x - d : threadIdx.x); }
static long __shfl_xor(long v, int d, int) { return exchange(v, threadIdx.x ^ d); }

namespace {
constexpr int C = DELTA_CHUNK, B = DELTA_BLOCK;
enum { NARROW = 0, ROWS = 1, FOURS = 2 };
%s
static DeltaArgs g_args;
static long g_work;
static void thread_main() {
  delta_plan_kernel(g_args, g_work);
  --g_left;
}
static hipError_t launch(void (*)(DeltaArgs, long), dim3, dim3 block, unsigned, hipStream_t, DeltaArgs a, long work) {
  static std::vector<char> stacks(PLAN * 16384);
  g_args = a, g_work = work, g_left = block.x;
  for (unsigned t = 0; t < block.x; ++t) {
    g_parity[t] = 0;
    getcontext(&g_thread[t]);
    g_thread[t].uc_stack.ss_sp = stacks.data() + t * 16384;
    g_thread[t].uc_stack.ss_size = 16384;
    g_thread[t].uc_link = &g_main;
    makecontext(&g_thread[t], thread_main, 0);
  }
  while (g_left == (int)block.x)
    for (unsigned t = 0; t < block.x; ++t) {
      threadIdx.x = t;
      swapcontext(&g_main, &g_thread[t]);
    }
  if (g_left) abort();   // they parted
  return hipSuccess;
}
static void delta_zero_kernel(DeltaArgs) {}
static hipError_t launch(void (*)(DeltaArgs), dim3, dim3, unsigned, hipStream_t, DeltaArgs) { return hipSuccess; }
%s
}  // namespace

// The workgroups of a head: jobs (sequence, from, to, first, last) and blocks (row, count); what there is of either.
extern "C" int divide(size_t rows, size_t n, size_t heads, size_t dk, size_t dv, const long* begin, const long* end, int backward, long* job, int* jobs,
                      long* block, int* blocks) {
  DeltaArgs a = {};
  a.rows = rows, a.n_seq = n, a.heads = (int)heads, a.key_heads = (int)heads, a.dk = (int)dk, a.dv = (int)dv;
  a.begin = begin, a.end = end, a.index_bytes = 8;
  const size_t bytes = sizes_of(rows, n, heads, heads, dk, dv, backward).bytes;
  // nothing but the plan's own parts is touched, at its beginning
  std::vector<char> ws(bytes < (1u << 22) ? bytes : (1u << 22));
  memset(ws.data(), 0x3f, ws.size());
  a.workspace = ws.data();
  lay_out(a, backward);
  if (plan(a, nullptr) != hipSuccess) return -1;
  const size_t launched = a.segments ? a.segments : a.n_seq;
  *jobs = *blocks = 0;
  for (size_t i = 0; i < launched; ++i) {
    Job w;
    if (!find_job(a, i, w)) continue;
    const long found[5] = {(long)w.s, w.from, w.to, w.first, w.last};
    memcpy(job + 5 * (*jobs)++, found, sizeof found);
  }
  for (size_t i = 0; i < a.blocks; ++i) {
    Block w;
    if (!find_block(a, i, w)) continue;
    block[2 * *blocks] = w.row, block[2 * *blocks + 1] = w.count;
    ++*blocks;
  }
  return 0;
}

// The places of a head's segments, and how many there are; -1: a job that is cut has none behind or in front of it.
extern "C" long places(size_t rows, size_t n, size_t heads, const long* begin, const long* end, long* place, int* count) {
  DeltaArgs a = {};
  a.rows = rows, a.n_seq = n, a.heads = a.key_heads = (int)heads, a.dk = a.dv = 128;
  a.begin = begin, a.end = end, a.index_bytes = 8;
  const Sizes sizes = sizes_of(rows, n, heads, heads, 128, 128, false);
  std::vector<char> ws(sizes.matrices);
  memset(ws.data(), 0x3f, ws.size());
  a.workspace = ws.data();
  lay_out(a, false);
  if (plan(a, nullptr) != hipSuccess) return -1;
  const size_t launched = a.segments ? a.segments : a.n_seq;
  *count = 0;
  for (size_t i = 0; i < launched; ++i) {
    Job w;
    if (find_job(a, i, w) && !(w.first && w.last)) place[(*count)++] = (long)w.slot;
  }
  if (sizes.maps - sizes.fronts < sizes.slots * heads * 128 * 128 * 4 || sizes.bytes - sizes.maps < sizes.slots * heads * 128 * 128 * 4) return -1;
  return (long)sizes.slots;
}
"""


def section(text, begin, end):
    return text[text.index(begin):text.index(end, text.index(begin))]


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    csrc = os.path.join(build.HERE, "csrc")
    shared, text = (open(os.path.join(csrc, f)).read() for f in ("amp_ops.h", "amp_delta.hip"))
    device = (section(text, "// ------------------------------------------------------------------ where things are", "// N and P of a chunk") +
              section(text, "// ------------------------------------------------------------------ plan", "// Rows of no sequence"))
    # 256 threads, the fewest that the order takes, and what the plan keeps near in either place
    few = "PLAN = 1024, NEAR = 4096"
    assert few in device
    device = device.replace(few, "PLAN = 256, NEAR = 64")
    host = section(text, "struct Sizes", "template <class T, int KT>\nhipError_t prepare")
    tmp = tmp_path_factory.mktemp("plan")
    src, so = tmp / "p.cpp", tmp / "p.so"
    src.write_text(HOST % (section(shared, "#define DELTA_CHUNK", "struct DeltaStepArgs"), device, host))
    p = subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-std=c++17", "-w", str(src), "-o", str(so)], stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout
    return ct.CDLL(str(so))


def divide(lib, rows, begin, end, heads, dk, dv, backward=0):
    n = 1 if begin is None else len(begin)
    most = rows // 64 + min(n, rows)
    job, block, counts = np.zeros((most + n, 5), np.int64), np.zeros((most + 1, 2), np.int64), np.zeros(2, np.int32)
    at = lambda x: None if x is None else ct.c_void_p(x.ctypes.data)  # noqa: E731
    if begin is not None:
        begin, end = (np.ascontiguousarray(np.append(x, 0), np.int64) for x in (begin, end))   # an address without sequences too
    size = ct.c_size_t
    assert lib.divide(size(rows), size(n), size(heads), size(dk), size(dv), at(begin), at(end), backward, at(job), at(counts[:1]), at(block),
                      at(counts[1:])) == 0
    return job[:counts[0]], block[:counts[1]]


def check(lib, rows, begin, end, heads, dk=128, dv=128, backward=0):
    """Every sequence's blocks once, in jobs of which one is its first and one its last."""
    job, block = divide(lib, rows, begin, end, heads, dk, dv, backward)
    spans = [(0, rows)] if begin is None else list(zip(begin, end))
    want = [(r, min(64, e - r)) for b, e in spans for r in range(b, e, 64)]
    assert sorted(map(tuple, block.tolist())) == sorted(want)
    cut = 0
    by = {}
    for s, a, b, first, last in job.tolist():
        by.setdefault(s, []).append((a, b, first, last))
    assert sorted(by) == list(range(len(spans))), (rows, heads)
    for s, (b, e) in enumerate(spans):
        parts = sorted(by[s])
        at = [p[0] for p in parts] + [(e - b + 63) // 64]
        assert at[0] == 0 and [p[1] for p in parts] == at[1:], (rows, heads, parts)
        assert [p[2] for p in parts] == [1] + [0] * (len(parts) - 1), (rows, heads, parts)
        assert [p[3] for p in parts] == [0] * (len(parts) - 1) + [1], (rows, heads, parts)
        cut += len(parts) > 1
    return cut


@pytest.mark.parametrize("heads,dv", [(1, 20), (1, 128), (2, 64), (4, 130), (8, 128), (16, 128), (32, 64)])
def test_one_sequence_without_bounds(library, heads, dv):
    cut = 0
    for rows in list(range(0, 130)) + [64 * k + d for k in range(20, 140) for d in (-1, 0, 1)] + [16384, 32768, 65536, 1 << 20]:
        cut += check(library, rows, None, None, heads, 128, dv)
        if rows % 640 == 0:   # and as offsets say it
            assert (divide(library, rows, None, None, heads, 128, dv)[0] == divide(library, rows, [0], [rows], heads, 128, dv)[0]).all()
    assert cut


def packed(lengths, gaps=None):
    at, begin, end = 0, [], []
    for i, n in enumerate(lengths):
        at += gaps[i] if gaps else 0
        begin.append(at)
        at += n
        end.append(at)
    return begin, end, at


@pytest.mark.parametrize("heads", [1, 4, 16])
def test_sequences_by_their_bounds(library, heads):
    rng = np.random.default_rng(heads)
    cut = 0
    for lengths in ([2000, 0, 3, 2300], [64 * 32], [64 * 24, 64 * 48], [0, 0, 5], [1], [64] * 30, [5] * 70, [4096] + [1] * 300, [0] * 5 + [3000] + [0] * 5,
                    *(rng.integers(0, 3000, rng.integers(1, 12)).tolist() for _ in range(12))):
        begin, end, rows = packed(lengths)
        cut += check(library, rows, begin, end, heads)
        begin, end, rows = packed(lengths, rng.integers(0, 70, len(lengths)).tolist())
        cut += check(library, rows + 50, begin, end, heads, 33, 40, 1)
    assert cut
    check(library, 10, [], [], heads)


def places(lib, rows, begin, end, heads):
    n = 1 if begin is None else len(begin)
    place, count = np.zeros(rows // 64 + 2 * n, np.int64), np.zeros(1, np.int32)
    at = lambda x: None if x is None else ct.c_void_p(x.ctypes.data)  # noqa: E731
    if begin is not None:
        begin, end = (np.ascontiguousarray(x, np.int64) for x in (begin, end))
    size, lib.places.restype = ct.c_size_t, ct.c_long
    there = lib.places(size(rows), size(n), size(heads), at(begin), at(end), at(place), at(count))
    assert there >= 0
    return there, place[:count[0]].tolist()


def test_segments_of_sequences_that_are_cut_have_places(library):
    """A place to each, one behind the other, within the workspace; sequences out of order, whose segments would be too many, are not cut."""
    rng = np.random.default_rng(3)
    cut = 0
    for lengths in ([64 * 24], [1537], [2000, 0, 3, 2300], [513] * 2 + [1600], [40] * 100 + [2200, 577, 576] + [3] * 70,
                    *(rng.integers(0, 4000, rng.integers(1, 12)).tolist() for _ in range(20))):
        begin, end, rows = packed(lengths)
        there, got = places(library, rows, begin, end, 1)
        assert got == list(range(len(got))) and len(got) <= there
        cut += bool(got)
        there, got = places(library, rows, None, None, 1)
        assert got == list(range(len(got))) and len(got) <= there
    assert cut > 10
    for rows in (1536, 4000, 70000):
        for n in (2, 5, 300):
            there, got = places(library, rows, [0] * n, [rows] * n, 1)
            assert got == list(range(len(got))) and len(got) <= there


def test_workspace_of_short_sequences():
    """Nothing for segments but what sequences that are cut could take: of 1,000 times 20 rows, a place to 256 of the rows."""
    from paper_1705_09786_amd import binding as B
    shape, n = B.DeltaShape(B.BF16, 20000, 16, 16, 128, 128), ct.c_size_t()
    assert B.lib().amp_gated_delta_workspace(shape, 1000, 0, ct.byref(n)) == B.AMP_OK
    blocks, state = (20000 // 64 + 1000) * 16, 128 * 128 * 4
    own = blocks * (4 * 32 * 32 * 4 + 4 * 64 * 4 + 64 * 8)   # N and P, powers, sums of decays
    assert n.value <= own + 20000 // 256 * 16 * 2 * state + 100000
