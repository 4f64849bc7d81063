"""The order in which psrl_kv_move's large moves store their parts, as a model on the CPU.

csrc/move_order.h holds the arithmetic: which groups of parts a part waits for, which groups a warp looks at, the count at
which a group is complete (counts are kept modulo a ring and never reset).  The model here compiles that header, hands parts
out in order to as many warps as the kernel has, lets every step take a random time - some of them very long, some warps
starting very late - and checks at every store that nothing it overwrites has yet to be loaded.  A GPU without other work
hardly ever delays a warp like that, so a test there would not see a hole."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2608_25683_b200 import build

MODEL = r"""
#include <algorithm>
#include <cstdlib>
#include <queue>
#include <random>
#include <vector>
#include "move_order.h"
using namespace psrl;

struct List { int32_t n, slots; const int32_t *src, *dst, *first; };

// out: parts, stores before a source was loaded, stores whose groups were not all complete, 1 if everything was stored
extern "C" void run(int n, const int32_t* src, const int32_t* dst, const int32_t* first, int heads, uint32_t part_rows, int warps,
                    uint32_t seed, double long_share, double long_time, int late_warps, double late_time, int64_t* out) {
  const List list{n, first[n], src, dst, first};
  const uint32_t rows = uint32_t(list.slots) * heads, n_parts = (rows + part_rows - 1) / part_rows;
  // the parts whose sources a part overwrites: a range for each, as destinations and sources both ascend
  std::vector<std::vector<uint32_t>> over(n_parts);
  for (int e = 0; e < n; ++e)
    for (int i = 0; i < first[e + 1] - first[e]; ++i) {
      const int d = dst[e] + i, x = extent_of(src, n, d);
      if (src[x] > d || d - src[x] >= first[x + 1] - first[x]) continue;   // nobody's source
      for (int h = 0; h < heads; ++h) {
        const uint32_t row = uint32_t(h) * list.slots + first[e] + i, victim = uint32_t(h) * list.slots + first[x] + d - src[x];
        auto& o = over[row / part_rows];
        if (o.empty() || o.back() != victim / part_rows) o.push_back(victim / part_rows);
      }
    }
  std::mt19937 rng(seed);
  auto rnd = [&] { return std::uniform_real_distribution<double>(0, 1)(rng); };
  auto takes = [&](double t) { return t * (0.8 + 0.4 * rnd()) * (rnd() < long_share ? long_time : 1.0); };
  std::vector<char> loaded(n_parts, 0);
  std::vector<uint32_t> groups((n_parts + kGroup - 1) / kGroup, 0);
  uint32_t ring[kRing] = {}, next_part = 0, stored = 0;
  int64_t early = 0, unseen = 0;
  enum Step { kTake, kLoaded, kPoll };
  struct Warp { Step step; uint32_t part, seen; };
  std::vector<Warp> w(warps, Warp{kTake, 0, 0});
  struct Event { double at; int warp; bool operator<(const Event& o) const { return at > o.at; } };
  std::priority_queue<Event> q;
  for (int i = 0; i < warps; ++i) q.push({(i < late_warps ? late_time : 1.0) * rnd(), i});
  double end_of_time = 1e7;
  while (!q.empty() && q.top().at < end_of_time) {
    const Event ev = q.top();
    q.pop();
    Warp& x = w[ev.warp];
    if (x.step == kTake) {
      if (next_part == n_parts) continue;
      x.part = next_part++;
      x.step = kLoaded;
      q.push({ev.at + takes(1.0), ev.warp});
    } else if (x.step == kLoaded) {
      loaded[x.part] = 1;
      ++groups[x.part / kGroup];
      ++ring[x.part / kGroup % kRing];
      x.step = kPoll;
      q.push({ev.at + 0.02, ev.warp});
    } else {
      const uint32_t group = x.part / kGroup, until = wait_until(list, x.part, std::min((x.part + 1) * part_rows, rows), part_rows);
      const uint32_t from = poll_from(x.seen, group);
      bool ok = true;
      for (uint32_t lane = 0; lane < 32; ++lane)
        if (from + lane <= until && ring[(from + lane) % kRing] < full_count(from + lane, n_parts)) ok = false;
      if (!ok) { q.push({ev.at + 0.02, ev.warp}); continue; }
      x.seen = std::max(x.seen, until + 1);
      bool bad = false;
      for (uint32_t o : over[x.part]) bad |= !loaded[o];
      early += bad;
      bad = false;
      for (uint32_t g = 0; g <= until; ++g) bad |= groups[g] < std::min(kGroup, n_parts - g * kGroup);
      unseen += bad;
      ++stored;
      x.step = kTake;
      q.push({ev.at + takes(1.0), ev.warp});
    }
  }
  out[0] = n_parts; out[1] = early; out[2] = unseen; out[3] = stored == n_parts;
}
"""


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    where = tmp_path_factory.mktemp("move_order")
    source, lib = where / "model.cpp", where / "model.so"
    source.write_text(MODEL)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC, str(source), "-o", str(lib)])
    fn = ctypes.CDLL(str(lib)).run
    ip = np.ctypeslib.ndpointer(np.int32, flags="C")
    fn.argtypes = [ctypes.c_int, ip, ip, ip, ctypes.c_int, ctypes.c_uint32, ctypes.c_int, ctypes.c_uint32, ctypes.c_double, ctypes.c_double,
                   ctypes.c_int, ctypes.c_double, np.ctypeslib.ndpointer(np.int64, flags="C")]

    def run(extents, heads, part_rows, seed, warps=444, long_share=0.0, long_time=1.0, late_warps=0, late_time=1.0):
        e = np.asarray(extents, dtype=np.int64)
        src, dst = (np.ascontiguousarray(e[:, i], dtype=np.int32) for i in (0, 1))
        first = np.concatenate([[0], np.cumsum(e[:, 2])]).astype(np.int32)
        out = np.zeros(4, dtype=np.int64)
        fn(len(e), src, dst, first, heads, part_rows, warps, seed, long_share, long_time, late_warps, late_time, out)
        return dict(zip(("parts", "early", "unseen", "done"), out.tolist()))

    return run


def arena(n, lo, hi, hole, seed, big_hole=0):
    """Moves of a compaction; with big_hole the first blocks of the arena were freed, so that a head begins with displacements
    of that many slots."""
    rng = np.random.default_rng(seed)
    size = 16 * rng.integers(lo // 16, hi // 16 + 1, n)
    gap = 16 * rng.binomial(1, hole, n) * rng.integers(1, hi // 16 + 1, n)
    gap[0] = max(16, big_hole)
    src = np.cumsum(size + gap) - size
    return np.stack([src, np.cumsum(size) - size, size], 1)


@pytest.mark.parametrize("kind", ["tenth", "half", "big displacements", "one slot"])
@pytest.mark.parametrize("delays", [dict(), dict(long_share=0.001, long_time=5), dict(long_share=0.002, long_time=40),
                                    dict(late_warps=30, late_time=60), dict(late_warps=200, late_time=20, long_share=0.001, long_time=8)])
def test_no_part_is_stored_too_early(model, kind, delays):
    extents = {"tenth": lambda s: arena(150, 64, 1024, 0.1, s), "half": lambda s: arena(150, 64, 1024, 0.5, s),
               "big displacements": lambda s: arena(100, 64, 1024, 0.1, s, big_hole=30000),
               "one slot": lambda s: np.array([[1, 0, 70000 + s]])}[kind]
    for seed in range(3):
        got = model(extents(seed), 16, 256, seed, **delays)
        assert got["parts"] > 3 * 32 * 32 and got["done"]          # the ring goes round several times
        assert got["early"] == 0 and got["unseen"] == 0, got


@pytest.mark.parametrize("warps", [32, 96, 480])
def test_few_warps_and_short_moves_end(model, warps):
    """The smallest grid that may run, and fewer parts than a group: every wait ends."""
    for n, heads in ((1, 1), (3, 2), (40, 8)):
        got = model(arena(n, 64, 512, 0.3, n), heads, 256, 5, warps=warps, long_share=0.01, long_time=30)
        assert got["done"] and got["early"] == 0 and got["unseen"] == 0
