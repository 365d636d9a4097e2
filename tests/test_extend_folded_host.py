"""Slots of a folded group's own pages that hold no key: which they are, compiled for the host, against the rows' keys one by one. What lies in
them is zeroed without a further look; a slot that counted as seen would have every row gone through again wherever it holds NaN."""
import ctypes
import random
import subprocess

import numpy as np
import pytest

from paper_2609_30884_gb300 import build
from tests.test_extend_wider_host import SHIM, ints

MORE = r"""
// Of every slot of the folded entries' own pages, in order of entries and pages: what the kernel says, and whether some row's keys hold it.
// Returns the slots.
extern "C" int own_slots(int* says, int* holds, int most) {
  const AttnTable& c = args.c;
  int n = 0;
  for (int i = 0; i < c.n; ++i) {
    if (c.members[i] == 0) continue;
    const KeyRange own = some_keys(c, i, 0, c.rows[i] - 1, args.d.causal, 0);
    for (int key = own.lo; key < own.hi; ++key, ++n) {
      if (n >= most) return -1;
      const int at = key - own_key0(c, i);
      says[n] = own_slot_seen(c, i, at / kPage, at % kPage, args.d.causal);
      holds[n] = 0;
      for (int r = 0; r < c.rows[i]; ++r) {
        const KeyRange k = folded_row(c, i, r, args.d.causal);
        holds[n] |= key >= k.lo && key < k.hi;
      }
    }
  }
  return n;
}
"""


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("folded")
    (d / "shim.cu").write_text(SHIM + MORE)
    subprocess.run([nvcc, *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.CSRC, "-I", build.INCLUDE,
                    "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", str(d / "shim.cu"), "-o", str(d / "plan.so")], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def slots(so, reqs, hq, hkv, groups, causal=True):
    """reqs: (rows, position, keys); groups: (requests, shared keys). Slots of the folded groups' own pages, those with a key."""
    n, pages = len(reqs), max(1, (max(r[2] for r in reqs) + 15) // 16)
    tables, info = np.zeros((n, pages), dtype=np.int32), (ctypes.c_int * 7)()
    spare = (ctypes.c_int * 100000)()
    so.make(n, ints([r[0] for r in reqs]), ints([r[1] for r in reqs]), ints([r[2] for r in reqs]), tables.ctypes.data_as(ctypes.c_void_p), pages,
            len(groups), ints([g[0] for g in groups]), ints([g[1] for g in groups]), hq, hkv, int(causal), 0, 0, 152, 0, info, spare, spare)
    says, holds = np.zeros(200000, dtype=np.int32), np.zeros(200000, dtype=np.int32)
    m = so.own_slots(says.ctypes.data_as(ctypes.c_void_p), holds.ctypes.data_as(ctypes.c_void_p), len(says))
    assert m >= 0 and np.array_equal(says[:m], holds[:m])
    return m, int(holds[:m].sum())


CASES = [
    ([(1, 900 + i, 901 + i) for i in range(8)], 4, 2, [(8, 900)]),                       # shared keys in the first page, slots behind the last key
    ([(1, 927 + i, 928 + i) for i in range(20)], 28, 4, [(20, 896)]),                     # first pages without shared keys
    ([(5, 400, 405)] * 6 + [(3, 700, 703)] * 4, 12, 2, [(6, 400), (4, 555)]),
    ([(1, 300, 301), (0, 0, 0), (1, 350, 351), (4, 300, 304), (0, 9, 9)], 4, 2, [(5, 300)]),  # requests without rows
    ([(3, 1900, 5000)] * 4 + [(3, 1900, 2100)] * 3, 28, 4, [(7, 1900)]),                  # keys behind the rows
    ([(1, 500, 500)] * 3 + [(2, 510, 512)], 4, 2, [(4, 500)]),                             # some without keys of their own
    ([(64, 900, 964)] * 3 + [(1, 900, 901)] * 9, 4, 2, [(3, 900), (9, 900)]),              # rows that see one key more each
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_slots_without_a_key(planner, case, causal):
    reqs, hq, hkv, groups = CASES[case]
    n, held = slots(planner, reqs, hq, hkv, groups, causal)
    # (rows that see keys far behind them: such a group is split, and has no pages end to end)
    assert 0 < held < n or (n == 0 and not causal and case == 4)


def test_slots_without_a_key_of_random_groups(planner):
    rng, some = random.Random(7), 0
    for _ in range(60):
        hq, hkv = rng.choice(((4, 2), (7, 1), (3, 3), (16, 1)))
        reqs, groups = [], []
        for _ in range(rng.randint(1, 3)):
            count, shared = rng.randint(2, 9), rng.choice((1024, rng.randint(700, 2500)))
            groups.append((count, shared))
            for _ in range(count):
                m, extra = rng.choice((0, 1, 1, rng.randint(1, 30))), rng.choice((0, rng.randint(0, 90)))
                reqs.append((m, shared + extra, shared + extra + rng.choice((m, m, 0, rng.randint(0, m + 20)))))
        if any(r[0] for r in reqs):
            some += slots(planner, reqs, hq, hkv, groups, rng.random() < 0.8)[0] > 0
    assert some > 30
