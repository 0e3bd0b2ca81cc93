"""How the attention of new rows shares its work out, without a GPU: the workgroups that a launch starts and those that the
plan on the device counts on, by the functions of csrc/paged.h that both use, compiled by the host compiler."""
import ctypes
import subprocess

import numpy as np
import pytest

from tests.test_paged_host import CSRC

SRC = r"""
#include "%s/paged.h"
#include <vector>
using namespace uad;
// What a call of these starts and lengths comes to: units, workgroups and slots that the plan
// counts on, workgroups that the launch starts, its bound of the units.
static void plan(const RowsKind &k, bool cut, int n_rows, int n_seqs, const int *starts, const int *lens, int hkv, int group, int pages, int shift,
                 int window, int sinks, int target, long long *o) {
  const RowsGrid grid = rows_grid(k, n_rows, n_seqs, true, hkv, group, cut ? (int64_t)pages << shift : k.tile, window, sinks, target, max_slots(target));
  int64_t tiles = 0;
  int units = 0, wgs = 0, slots = 0;
  bool falls = false;
  std::vector<SeenTiles> seen;
  std::vector<int> of;
  for (int b = 0; b < n_seqs; ++b) {
    const bool ok = sequence_ok(b, starts[b], starts[b + 1], n_rows, lens[b], pages, shift);
    falls |= starts[b] > starts[b + 1];
    const int n = ok ? starts[b + 1] - starts[b] : 0, len = ok ? lens[b] : 0;
    of.push_back(hkv * runs_of(n, group, k.cols));
    seen.push_back(seen_tiles(len, seen_from(len - n, window), sinks, k.tile));
    units += of[b];
    tiles += (int64_t)of[b] * seen[b].count;
  }
  auto count = [&](int share) {
    wgs = 0;
    for (int b = 0; b < n_seqs; ++b) wgs += rows_splits(k, seen[b].count, share) * of[b];
    return wgs;
  };
  const int share = rows_share(k, grid.unsplit || falls ? kUncut : first_share(tiles, target, k.min_tiles), units, target, count);
  for (int b = 0; b < n_seqs; ++b) {
    const int s = rows_splits(k, seen[b].count, share);
    if (s > 1) slots += s * of[b];
  }
  o[0] = units, o[1] = wgs, o[2] = slots, o[3] = grid.wgs;
  o[4] = hkv * ((int64_t)n_rows * group / k.cols + n_seqs);
}
extern "C" void plan_of(const int *kind, int one_round, int cut, int n_rows, int n_seqs, const int *starts, const int *lens, int hkv, int group,
                        int pages, int shift, int window, int sinks, int target, long long *o) {
  plan(RowsKind{kind[0], kind[1], kind[2], kind[3], one_round != 0}, cut != 0, n_rows, n_seqs, starts, lens, hkv, group, pages, shift, window, sinks, target, o);
}
// Mixes whose units are `runs` of each KV head: how many of them have splits, and how many a
// launch that is too small (or slots that are too few).
extern "C" void mixes(unsigned seed, int n, const int *kind, int one_round, int cut, int runs, int hkv, int group, int target, int *split, int *bad, int *at_bound) {
  const RowsKind k{kind[0], kind[1], kind[2], kind[3], one_round != 0};
  uint64_t state = seed * 2654435761u + 88172645463325252ull;
  auto below = [&](int m) {
    state ^= state << 13, state ^= state >> 7, state ^= state << 17;
    return (int)((state >> 11) %% (unsigned)m);
  };
  *split = *bad = *at_bound = 0;
  for (int i = 0; i < n; ++i) {
    const int most = runs < 90 ? runs : 90, seqs = 1 + below(below(3) ? (most < 6 ? most : 6) : most);
    std::vector<int> r(seqs, 1), starts(1, 0), lens;
    for (int left = runs - seqs; left > 0;) {
      const int b = below(seqs), take = 1 + below(left);
      r[b] += take, left -= take;
    }
    const int window = below(3) ? 0 : 1 + below(3000), sinks = window && below(2) ? below(200) : 0, partly = below(3);
    for (int b = 0; b < seqs; ++b) {
      // rows of r[b] units of a KV head: the fewest, or any
      const int least = (int)((int64_t)(r[b] - 1) * k.cols / group) + 1, largest = (int)((int64_t)r[b] * k.cols / group);
      const int rows = least >= largest || partly ? least : least + below(largest - least + 1);
      starts.push_back(starts.back() + rows);
      lens.push_back(rows + (below(2) ? 0 : below(2) ? below(500) : below(60000)));
    }
    long long o[5];
    plan(k, cut != 0, starts.back() + (below(4) ? 0 : below(50)), seqs, starts.data(), lens.data(), hkv, group, 1 << 14, 4 + below(5), window, sinks, target, o);
    *split += o[2] > 0;
    *at_bound += o[4] == target;
    *bad += o[1] > o[3] || o[2] > max_slots(target);
  }
}
"""

# tile, columns of a unit, whole, least tiles of a split; and whether all fit one round, and are split at all
FEW = [((32, 16, w, 4), 0, 1) for w in (8, 12, 20)] + [((64, 16, w, 4), 0, 1) for w in (6, 9, 15)]
MANY = [((64, 64, 6, 3), 1, 1), ((64, 128, 6, 3), 1, 0)]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "p.cpp").write_text(SRC % CSRC)
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    return ctypes.CDLL(str(d / "p.so"))


def ints(x):
    return (ctypes.c_int * len(x))(*x)


def plan(lib, kind, new, lens, hkv, group, target, starts=None, n_rows=None, window=0, sinks=0):
    """Units, workgroups and slots that the plan counts on, workgroups that are launched."""
    (k, one_round, cut), o = kind, (ctypes.c_longlong * 5)()
    starts = [0, *map(int, np.cumsum(new))] if starts is None else starts
    lib.plan_of(ints(k), one_round, cut, max(starts) if n_rows is None else n_rows, len(lens), ints(starts), ints(lens), hkv, group, 1 << 12, 6, window, sinks,
                target, o)
    return o[0], o[1], o[2], o[3]


@pytest.mark.parametrize("new,lens,hkv,group,target", [
    ([10, 483], [3000, 483], 8, 4, 256), ([10, 481], [3000, 481], 8, 4, 256), ([241, 241], [10000, 241], 8, 4, 256), ([1, 2033], [4000, 2033], 1, 8, 256),
    ([10, 995], [3000, 995], 8, 4, 512), ([385, 609], [19200, 609], 4, 4, 256), ([65, 65, 65, 257], [30000, 65, 65, 257], 8, 4, 256)])
def test_as_many_units_as_run_at_once(lib, new, lens, hkv, group, target):
    units, wgs, slots, grid = plan(lib, MANY[0], new, lens, hkv, group, target)
    assert units == target and wgs <= grid and slots <= 2 * target


@pytest.mark.parametrize("kind", FEW + MANY)
@pytest.mark.parametrize("n_seqs,rows", [(5, 200), (5, 483), (90, 100), (3, 90)])
def test_starts_that_fall_leave_units_whole(lib, kind, n_seqs, rows):
    """Starts 0, n, 0, n, ..: usable sequences have more rows in all than the call, and the launch is for the call's.  No unit
    has splits then, so none is begun whose others are missing."""
    starts, lens = [rows * (b % 2) for b in range(n_seqs + 1)], [10000] + [rows] * (n_seqs - 1)
    units, wgs, slots, _ = plan(lib, kind, None, lens, 8, 4, 256, starts=starts, n_rows=rows)
    assert slots == 0 and wgs == units == 8 * ((n_seqs + 1) // 2) * -(-rows * 4 // kind[0][1])


@pytest.mark.parametrize("kind", FEW + MANY)
@pytest.mark.parametrize("target", [256, 512, 304])
def test_what_the_plan_counts_on_is_launched(lib, kind, target):
    """Units at, below and above as many as run at once."""
    k, one_round, cut = kind
    splits = bounds = 0
    for seed, (hkv, group) in enumerate([(1, 8), (1, 3), (1, 40), (2, 4), (4, 1), (8, 4), (16, 16)]):
        for runs in {max(1, target // hkv + d) for d in (-2, -1, 0, 1, 2)} | {1, 2, 7, target // hkv // 2, 3 * target // hkv}:
            split, bad, at_bound = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
            lib.mixes(seed + runs, 400, ints(k), one_round, cut, runs, hkv, group, target, *map(ctypes.byref, (split, bad, at_bound)))
            assert bad.value == 0, (hkv, group, runs, bad.value)
            splits += split.value
            bounds += at_bound.value
    assert not cut or splits > 3000
    assert bounds > 300  # the launch's own bound of the units, too
