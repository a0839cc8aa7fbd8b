"""How the 8-bit attention cuts the steps of a call into ranges, on the host: the kernel's own
arithmetic (csrc/q8_ranges.h), compiled for the CPU."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_09603_amd", "csrc")
LIMIT = 1 << 30
WGS = 512  # 256 CUs

SOURCE = r"""
#include "q8_ranges.h"
using namespace echo;
// Requests with tiles[r] > 0 row tiles per head and units of tpu[r] steps: whether the call is refused, and of
// every place and wave (lo, hi, class, gang, member, its place's class's first place, their number).
extern "C" int cut(const int* tiles, const int* tpu, int R, int hkv, int wgs, int* out) {
  Q8Steps t;
  for (int r = 0; r < R; ++r) t.add(hkv, tiles[r], tpu[r]);
  int tot[kQ8Classes];
  for (int c = 0; c < kQ8Classes; ++c) tot[c] = int(t.of[c]);
  const bool refused = q8_refuses(t.all, tot);
  const float cost = q8_cost(tot, 0) + q8_cost(tot, 1) + q8_cost(tot, 2);
  for (int g = 0; g < wgs; ++g) {
    const Q8Share s = q8_share(tot, wgs, float(wgs) / cost, g);
    for (int w = 0; w < kQ8Waves; ++w) {
      const Q8Range x = q8_range_at(s, tot[s.cls], g, w);
      const int v[7] = {x.lo, x.hi, s.cls, x.gang, x.member, x.wg0, x.nwg};
      for (int i = 0; i < 7; ++i) *out++ = v[i];
    }
  }
  return refused ? 1 : 0;
}
extern "C" int range_of(int steps, int gangs, int older, int t) { return Q8Cutter(steps, gangs, older).range_of(t); }
extern "C" int first(int steps, int gangs, int older, int g) { return Q8Cutter(steps, gangs, older).first(g); }
extern "C" int unit_steps(int nslots, int P) { return q8_unit_steps(nslots, P); }
extern "C" int passes(int tiles, int c) { return q8_passes(tiles, c); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("ranges")
    src, so = str(d / "ranges.cpp"), str(d / "ranges.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    # (wrapping sums: what overflows is to be seen in the ranges, not left to the optimiser)
    subprocess.run([cxx, "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so],
                   check=True)
    return ctypes.CDLL(so)


def _cut(lib, requests, hkv, wgs=WGS):
    """requests: (row tiles per head, steps of a unit).  Whether the call is refused, and the
    ranges [wgs * 4, 7]."""
    t = np.ascontiguousarray([[a for a, _ in requests], [b for _, b in requests]], np.int32)
    out = np.zeros((wgs * 4, 7), np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    return bool(lib.cut(p(t[0]), p(t[1]), len(requests), hkv, wgs, p(out))), out


def _passes(tiles, c):
    """A head's rows go to gangs of four, what is left to one of one, two or (three) four."""
    rest = tiles % 4
    return (tiles // 4 + (rest == 3)) if c == 2 else int(rest == c + 1)


def _totals(requests, hkv):
    return [sum(hkv * tpu * _passes(tiles, c) for tiles, tpu in requests) for c in range(3)]


def _covered(out, tot):
    """Every step of every class is in the range of one gang, all of whose waves have it."""
    busy = out[out[:, 0] < out[:, 1]]
    assert np.all(busy[:, 0] >= 0)
    for c in range(3):
        of = busy[busy[:, 2] == c]
        if tot[c] == 0:
            assert len(of) == 0
            continue
        gangs = {}
        for lo, hi, _, gang, member, wg0, nwg in of.tolist():
            gangs.setdefault(gang, []).append((lo, hi, member))
            assert nwg > 0 and 0 <= wg0 and wg0 + nwg <= WGS
        at = 0
        for gang in range(len(gangs)):
            waves = gangs[gang]
            assert sorted(m for _, _, m in waves) == list(range(1 << c))
            assert len({(lo, hi) for lo, hi, _ in waves}) == 1 and waves[0][0] == at
            at = waves[0][1]
        assert at == tot[c]


@pytest.mark.parametrize("seed", range(40))
def test_ranges_cover_every_step_once(lib, seed):
    rng = np.random.default_rng(seed)
    R = int(rng.choice([1, 1, 2, 5, 40, 300]))
    hkv = int(rng.choice([1, 1, 2, 8, 40]))
    top = int(rng.choice([2, 30, 600, 40000]))
    kinds = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 33], size=int(rng.integers(1, 4)))
    requests = [(int(rng.choice(kinds)), int(rng.integers(1, top + 1))) for _ in range(R)]
    refused, out = _cut(lib, requests, hkv)
    assert not refused
    _covered(out, _totals(requests, hkv))


def test_a_small_class_beside_a_large_one(lib):
    """A class with little work has two workgroups at least, and long ranges therefore."""
    requests = [(1, 90)] * 900 + [(3, 90)]
    refused, out = _cut(lib, requests, 1)
    assert not refused
    _covered(out, _totals(requests, 1))
    of = out[(out[:, 2] == 2) & (out[:, 0] < out[:, 1])]
    assert set(of[:, 6]) == {2} and (of[:, 1] - of[:, 0]).max() > 32


# (row tiles, steps of a unit), KV heads: more than 2^30 steps in all
TOO_MANY = {
    "one class, 1.2e9": ([(1, 146485)] * 1024, 8),
    "2048 requests of 4 M tokens over shared pages, 8 heads": ([(1, 65539)] * 2048, 8),
    "1.8e9": ([(1, 219727)] * 1024, 8),
    "2.1e9": ([(1, 256348)] * 1024, 8),
    "gangs of two": ([(2, 150000)] * 1024, 8),
    "gangs of four": ([(4, 150000)] * 1024, 8),
    "gangs of four over the limit, others far below": ([(4, 150000)] * 1024 + [(1, 40)] * 9, 8),
    "all classes, each below the limit": ([(1, 60000), (2, 60000), (3, 60000)] * 1000, 8),
    "more than 2^32: the counts wrap to few": ([(1, 1 << 20)] * 4095 + [(1, (1 << 20) + 5)], 1 << 14),
    "2^33 in one request": ([(1, 1 << 25)], 256),
}


@pytest.mark.parametrize("name", sorted(TOO_MANY))
def test_more_steps_than_a_call_takes(lib, name):
    """Refused, and then no wave has a range, whatever the counts wrapped to."""
    requests, hkv = TOO_MANY[name]
    assert sum(_totals(requests, hkv)) > LIMIT
    refused, out = _cut(lib, requests, hkv)
    assert refused
    assert not out[:, :2].any()


@pytest.mark.parametrize("requests", [[(1, 1 << 17)] * 1024, [(2, 1 << 17)] * 1024, [(4, 1 << 17)] * 1024,
                                      [(1, 65000)] * 2000 + [(4, 70), (2, 3)]])
def test_as_many_steps_as_a_call_takes(lib, requests):
    refused, out = _cut(lib, requests, 8)
    assert not refused
    _covered(out, _totals(requests, 8))


@pytest.mark.parametrize("older", [17, 18])
@pytest.mark.parametrize("steps,gangs", [(1, 2), (2, 2), (3, 8), (7, 8), (1000, 2048), (4097, 2048), (99991, 512),
                                         (4_000_000, 2)])
def test_range_of_a_step(lib, steps, gangs, older):
    n = max(min(gangs, steps) // 2, 1)
    bounds = [lib.first(steps, gangs, older, g) for g in range(2 * n + 1)]
    assert bounds[0] == 0 and bounds[-1] == steps and sorted(bounds) == bounds
    for g in range(2 * n):
        if bounds[g] < bounds[g + 1]:
            for t in (bounds[g], bounds[g + 1] - 1):
                assert lib.range_of(steps, gangs, older, t) == g


def test_steps_of_a_unit(lib):
    for nslots in (1, 32, 33, 64, 65):
        for P in (0, 1, 63, 64, 65, 1 << 20, (1 << 31) - 1):
            assert lib.unit_steps(nslots, P) == 1 + -(-nslots // 32) + -(-P // 64)
    for tiles in range(1, 20):
        for c in range(3):
            assert lib.passes(tiles, c) == _passes(tiles, c)
