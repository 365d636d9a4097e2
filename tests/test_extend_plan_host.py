"""The host's plan of an attention call, without a GPU: the runs of the CTAs cover every item's steps once and in order, an
item that runs cut has its parts in slots of its own, and the workspace holds them. The plan's source is compiled into a
small library here; what it should say is derived from the rows' visible keys one by one."""
import ctypes
import random
import subprocess

import pytest

from paper_2609_30884_gb300 import abi, build
from tests.test_extend_host import A16, call_attention, chunks, ctx, lib, ref  # noqa: F401

TILE, CTAS = 128, 256  # rows of a query tile and keys of a K/V tile; CTAs at most
SUM = 128  # steps after which a sum starts anew

SHIM = r"""
#include "chunk_attn.cu"
namespace crf {  // what the launches need and the plan does not
PdlScope::PdlScope() : prev_(false) {}
PdlScope::~PdlScope() {}
bool pdl_active() { return false; }
}  // namespace crf
extern "C" size_t plan(int n, const int* n_new, const int* pos, const int* n_keys, int hq, int hkv, int dim, int causal,
                       int window, int sms, int* info, int* runs, int* rows, int* cuts) {
  crf::ChunkTable t = {};
  t.n = n;
  for (int i = 0; i < n; ++i) {
    t.row0[i + 1] = t.row0[i] + n_new[i];
    t.pos[i] = pos[i];
    t.n_keys[i] = n_keys[i];
  }
  static crf::ChunkPlan p;
  crf::plan_chunk_attention(t, hq, hkv, causal != 0, window, sms, &p);
  const int v[5] = {p.ctas, p.cuts, p.part_rows, p.merge_rows, p.longest};
  for (int i = 0; i < 5; ++i) info[i] = v[i];
  for (int i = 0; i <= p.ctas; ++i) {
    const int r[4] = {p.run[i].req, p.run[i].qt, p.run[i].g, p.run[i].step};
    for (int k = 0; k < 4; ++k) runs[4 * i + k] = r[k];
  }
  for (int i = 0; i <= p.cuts; ++i) rows[i] = p.rows[i];
  for (int i = 0; i < p.cuts; ++i) {
    const int c[6] = {p.cut[i].row0, p.cut[i].q0, p.cut[i].g, p.cut[i].first_slot, p.cut[i].cta, p.cut[i].parts};
    for (int k = 0; k < 6; ++k) cuts[6 * i + k] = c[k];
  }
  return crf::chunk_attention_workspace(p, dim);
}
"""


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cu").write_text(SHIM)
    subprocess.run([nvcc, *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.CSRC, "-I", build.INCLUDE,
                    "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", str(d / "shim.cu"), "-o", str(d / "plan.so")], check=True)
    so = ctypes.CDLL(str(d / "plan.so"))
    so.plan.restype = ctypes.c_size_t

    def plan(reqs, hq, hkv, dim, causal, window, sms):
        ints = lambda n: (ctypes.c_int * n)()  # noqa: E731
        cols = [(ctypes.c_int * len(reqs))(*c) for c in zip(*reqs)]
        info, runs, rows, cuts = ints(5), ints(4 * (CTAS + 1)), ints(CTAS + 1), ints(6 * CTAS)
        need = so.plan(len(reqs), *cols, hq, hkv, dim, int(causal), window, sms, info, runs, rows, cuts)
        ctas, n_cuts, part_rows, merge_rows, longest = info
        return dict(ctas=ctas, part_rows=part_rows, merge_rows=merge_rows, longest=longest, need=need, rows=list(rows)[:n_cuts + 1],
                    runs=[tuple(runs[4 * i:4 * i + 4]) for i in range(ctas + 1)],
                    cuts=[tuple(cuts[6 * i:6 * i + 6]) for i in range(n_cuts)])

    return plan


def items_of(reqs, hq, hkv, causal, window):
    """[(request, query tile, kv head, steps, first packed row, rows, first row of the request)] in the order of the runs."""
    grp, out, row0 = hq // hkv, [], 0
    for i, (m, pos, n) in enumerate(reqs):
        packed = m * grp
        tile, per = (TILE, 2) if packed <= TILE else (2 * TILE, 1)  # a step of few rows takes two K/V tiles
        for qt in reversed(range((packed + tile - 1) // tile)):
            q0, q1 = qt * tile, min(qt * tile + tile, packed)
            lo, hi = 1 << 60, 0
            for p in range(pos + q0 // grp, pos + (q1 - 1) // grp + 1):
                # keys that the rows of a tile see lie side by side, from its first row's first to its last one's last
                lo = min(lo, max(0, p - window + 1) if window else 0)
                hi = max(hi, min(n, p + 1) if causal else n)
            tiles = -(-hi // TILE) - lo // TILE if hi > lo else 0
            out += [(i, qt, g, -(-tiles // per), q0, q1 - q0, row0) for g in range(hkv)]
        row0 += m
    return out


def check(p, reqs, hq, hkv, dim, causal, window, sms):
    items = items_of(reqs, hq, hkv, causal, window)
    index = {(i, qt, g): k for k, (i, qt, g, *_) in enumerate(items)}
    assert p["ctas"] <= min(sms, CTAS) and p["runs"][-1] == (len(reqs), 0, 0, 0)
    if not items:
        assert p["ctas"] == 0 and p["need"] == 0
        return
    # starts in order, the first at the beginning, every one before its item's end: so the runs cover each step once
    starts = [(index[r[:3]], r[3]) for r in p["runs"][:-1]]
    assert starts[0] == (0, 0) and all(a < b for a, b in zip(starts, starts[1:]))
    assert all(s < items[k][3] or s == items[k][3] == 0 for k, s in starts)
    # items that a run starts inside of
    inside = {}
    for k, s in starts:
        if s:
            inside[k] = inside.get(k, 0) + 1
    want, used, rows = [], set(), [0]
    for k in sorted(inside):
        i, qt, g, steps, q0, n, row0 = items[k]
        cta = max(b for b, st in enumerate(starts) if st <= (k, 0))
        first = 2 * cta + (starts[cta] != (k, 0))
        want.append((row0, q0, g, first, cta, inside[k] + 1))
        # later parts open their CTA's run
        assert all(starts[cta + x][0] == k for x in range(1, inside[k] + 1))
        slots = [first] + [2 * (cta + x) for x in range(1, inside[k] + 1)]
        assert not used & set(slots) and max(slots) < 2 * p["ctas"]
        used |= set(slots)
        rows.append(rows[-1] + n)
    assert p["cuts"] == want and p["rows"] == rows and p["merge_rows"] == rows[-1]
    most = max((items[k][5] for k in inside), default=0)
    assert p["part_rows"] == most
    # every slot: a row's o, its maximum and its sum; and where a segment has more steps than a sum, both chains' totals
    ends = starts[1:] + [(len(items), 0)]
    longest = max(e - b for (k0, s0), (k1, s1) in zip(starts, ends) for k in range(k0, k1 + 1)
                  for b, e in [(s0 if k == k0 else 0, s1 if k == k1 else items[k][3])])
    assert p["longest"] == longest
    need = 4 * 2 * p["ctas"] * most * (dim + 2) + (4 * 2 * p["ctas"] * TILE * (dim + 2) if longest > SUM else 0)
    assert need <= p["need"] <= need + 512 and (p["need"] > 0) == (need > 0)


@pytest.mark.parametrize("seed", range(12))
def test_plans_of_random_calls(planner, seed):
    rng = random.Random(seed)
    spread = lambda a, b: int(round(a * (b / a) ** rng.random()))  # noqa: E731
    cut = 0
    for _ in range(60):
        hq, hkv, dim = rng.choice([(4, 2, 64), (12, 2, 128), (28, 4, 128), (5, 5, 64), (16, 1, 128), (200, 1, 64)])
        causal, window = rng.random() < 0.8, rng.choice((0, 0, 1, spread(1, 5000)))
        sms = rng.choice((1, 2, 8, 148, 152, 300))
        reqs = []
        for _ in range(rng.choice((1, 1, 2, 3, 8, 40, 128))):
            m, pos = rng.choice((0, 1, 1, spread(1, 20), spread(1, 900))), rng.choice((0, spread(1, 40), spread(1, 60000)))
            reqs.append((m, pos, rng.choice((pos + m, pos + m, pos + m, 0, spread(1, 70000)))))
        p = planner(reqs, hq, hkv, dim, causal, window, sms)
        check(p, reqs, hq, hkv, dim, causal, window, sms)
        cut += len(p["cuts"])
    assert cut > 0


def test_plans_of_empty_calls(planner):
    for reqs in ([(0, 5, 5)], [(0, 0, 0)] * 128, [(3, 10, 0)], [(700, 0, 0), (0, 9, 9)]):
        for sms in (1, 152):
            check(planner(reqs, 12, 2, 128, True, 0, sms), reqs, 12, 2, 128, True, 0, sms)


def test_attention_refuses_any_workspace_but_a_whole_one(lib, ctx):  # noqa: F811
    """One row over 100001 keys on 152 SMs is cut, so the call needs a workspace."""
    n, row = ctypes.c_size_t(), (1, 100000, 100001, A16)
    assert lib.crf_chunk_attention_workspace_size(ctx, 4, 2, 64, chunks(row), 1, 1, 0, ref(n)) == abi.OK
    assert n.value > 0 and n.value % 256 == 0
    assert call_attention(lib, ctx, ch=(row,), ws_bytes=n.value // 2) == abi.ENOMEM
    assert call_attention(lib, ctx, ch=(row,), ws_bytes=0) == abi.ENOMEM
    assert call_attention(lib, ctx, ch=(row,), ws=None) == abi.EINVAL
    assert call_attention(lib, ctx, ch=(row,), ws=A16 + 16) == abi.EINVAL
