"""Attention with sinks and over shared prefixes, as far as they go without a GPU: refusals, and the walk of every CTA through its
run. The kernel's plan, walk and tile ranges are compiled for the host; what they say is compared with the rows' visible
keys one by one: each row meets each of its keys exactly once, in a tile that its chain goes through and on a page that is
fetched, and no page without a visible key, nor any table entry behind the request's keys, is read."""
import ctypes
import random
import shutil
import subprocess

import numpy as np
import pytest

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300 import abi, build
from tests.test_extend_host import A16, HEADER, chunks, ctx, heads, lib, pool, ref  # noqa: F401

EINVAL, ESHAPE, EUNSUPPORTED, ENOMEM = abi.EINVAL, abi.ESHAPE, abi.EUNSUPPORTED, abi.ENOMEM
TILE, KEYS = 128, 128

SHIM = r"""
#include "chunk_attn_wider.cu"
namespace crf {  // what the launches need and the plan does not
PdlScope::PdlScope() : prev_(false) {}
PdlScope::~PdlScope() {}
bool pdl_active() { return false; }
}  // namespace crf
using namespace crf;
static ChunkArgs<true> args;
static AttnPlan plan;
static PrefixGroups groups;
static ChunkTable requests(int n, const int* n_new, const int* pos, const int* n_keys) {
  ChunkTable t = {};
  t.n = n;
  for (int i = 0; i < n; ++i) {
    t.row0[i + 1] = t.row0[i] + n_new[i];
    t.pos[i] = pos[i];
    t.n_keys[i] = n_keys[i];
    t.pt[i] = reinterpret_cast<const int32_t*>(static_cast<size_t>(16 * (i + 1)));
  }
  for (int i = n; i < kMaxChunks; ++i) t.row0[i + 1] = t.row0[n];
  return t;
}
// The plan; the number of CTAs. info: shared, entries, groups, items, part rows, cuts.
extern "C" int make(int n, const int* n_new, const int* pos, const int* n_keys, int n_groups, const int* count, const int* keys,
                    int hq, int hkv, int causal, int window, int sinks, int sms, int* info, int* of, int* firsts, int* lasts) {
  ChunkTable t = requests(n, n_new, pos, n_keys);
  memset(&args, 0, sizeof(args));
  AttnTable& a = args.c;
  if (n_groups) {
    share_prefixes(t, count, keys, n_groups, hq, hkv, &a, &groups);
  } else {
    groups.groups = 0;
    a.n = n;
    a.sinks = sinks;
    for (int i = 0; i < n; ++i) {
      a.row0[i] = t.row0[i], a.rows[i] = n_new[i], a.pos[i] = pos[i], a.n_keys[i] = n_keys[i], a.pt[i] = t.pt[i];
      groups.of[i] = -1;
    }
  }
  const bool shared = n_groups && groups.groups > 0;
  plan_attention(a, shared, hq, hkv, causal != 0, window, sms, &plan);
  memcpy(args.run, plan.runs.run, sizeof(args.run));
  args.d.n_q_heads = hq, args.d.n_kv_heads = hkv, args.d.causal = causal != 0, args.d.window = window;
  args.prefix.on = shared;
  args.prefix.first = firsts, args.prefix.last = lasts;
  memcpy(args.prefix.item0, plan.item0, sizeof(plan.item0));
  int row = 0;
  for (int b = 0; b < plan.runs.ctas; ++b) args.prefix.row0[b] = row, row += static_cast<int>(plan.run_rows[b]);
  const int v[6] = {shared, a.n, groups.groups, plan.items, static_cast<int>(plan.part_rows), plan.runs.cuts};
  memcpy(info, v, sizeof(v));
  for (int i = 0; i < n; ++i) of[i] = groups.of[i];
  return plan.runs.ctas;
}
extern "C" void table(int* row0, int* rows, int* pos, int* key0, int* n_keys, int* item0, int* pt) {
  for (int i = 0; i < args.c.n; ++i) {
    row0[i] = args.c.row0[i], rows[i] = args.c.rows[i], pos[i] = args.c.pos[i], key0[i] = args.c.key0[i];
    n_keys[i] = args.c.n_keys[i], item0[i] = plan.item0[i], pt[i] = static_cast<int>(reinterpret_cast<size_t>(args.c.pt[i]) / 16) - 1;
  }
}
// A CTA's segments, 26 numbers each; tiles: 11 each: cache tile, first and last page, and the ranges of what some row sees, what all rows
// of the two chains see. Returns the segments.
extern "C" int walk(int cta, int* seg, int* tiles, int max_tiles) {
  Walk<true> w;
  w.at = args.run[cta];
  w.part_row = args.prefix.row0[cta];
  int n = 0, m = 0;
  for (;; ++n) {
    SegmentOf<true> s;
    w.next(args, cta, s);
    if (s.end) return n;
    const int v[26] = {s.g, s.q0, s.rows, s.pos, s.n_keys, s.row0, s.narrow, s.slot, s.all_lo, s.all_hi, s.jb, s.J, s.n0, s.n1, s.quarters0,
                       s.quarters1, s.sinks, s.win_lo, s.ns, s.gap, s.part_row, s.item_rows, m,
                       static_cast<int>(reinterpret_cast<size_t>(s.pt) / 16) - 1, 0, 0};
    memcpy(seg + 26 * n, v, sizeof(v));
    const PageSpan<true> pages(s);
    for (int j = 0; j < s.J; ++j, ++m) {
      if (m >= max_tiles) return -1;
      const KeyRange all = range_in(s, j, KeyRange{s.all_lo, s.all_hi}), f0 = range_in(s, j, s.full0), f1 = range_in(s, j, s.full1);
      const int t[11] = {cache_tile(s, j), pages.first(j), pages.last(j), all.lo, all.hi, f0.lo, f0.hi, f1.lo, f1.hi, s.jb + j < s.ns, 0};
      memcpy(tiles + 11 * m, t, sizeof(t));
    }
  }
}
"""


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("wider")
    (d / "shim.cu").write_text(SHIM)
    subprocess.run([nvcc, *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.CSRC, "-I", build.INCLUDE,
                    "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", str(d / "shim.cu"), "-o", str(d / "plan.so")], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def ints(v):
    return (ctypes.c_int * max(1, len(v)))(*v)


def verify(so, reqs, hq, hkv, causal=True, window=0, sinks=0, groups=(), sms=152):
    """reqs: (rows, position, keys); groups: (requests, shared keys). Whether the call shares anything."""
    n, grp = len(reqs), hq // hkv
    info, of = (ctypes.c_int * 6)(), (ctypes.c_int * max(1, n))()
    firsts, lasts = (ctypes.c_int * 100000)(*[-1] * 100000), (ctypes.c_int * 100000)(*[-1] * 100000)
    ctas = so.make(n, ints([r[0] for r in reqs]), ints([r[1] for r in reqs]), ints([r[2] for r in reqs]), len(groups),
                   ints([g[0] for g in groups]), ints([g[1] for g in groups]), hq, hkv, int(causal), window, sinks, sms, info, of, firsts, lasts)
    shared, entries, n_groups, items, part_rows, cuts = info
    assert 0 < ctas <= sms and cuts <= 256
    tab = [(ctypes.c_int * entries)() for _ in range(7)]
    so.table(*tab)
    row0, rows, pos, key0, n_keys, item0, tables = ([int(x) for x in t] for t in tab)
    first_row = np.cumsum([0] + [r[0] for r in reqs])
    total = int(first_row[-1]) * hq
    longest = max(r[2] for r in reqs)
    met = np.zeros((total, longest), dtype=np.int32)  # (output row, head) x key, all entries' keys in the request's own numbering
    part_of = {}  # item -> [(part row, rows)], in order of runs
    seg, tiles = (ctypes.c_int * (26 * 4000))(), (ctypes.c_int * (11 * 60000))()
    slots, next_part = set(), 0
    for c in range(ctas):
        count = so.walk(c, seg, tiles, 60000)
        assert 0 <= count < 4000
        for k in range(count):
            (g, q0, packed, p, nk, r0, narrow, slot, all_lo, all_hi, jb, J, n0, n1, quarters0, quarters1, sk, win_lo, ns, gap, part_row, item_rows,
             m, table, _, _) = seg[26 * k:26 * k + 26]
            (e,) = [i for i in range(entries) if rows[i] and row0[i] == r0 and pos[i] == p and n_keys[i] == nk and tables[i] == table and rows[i] * grp == packed]
            tile = TILE if packed <= TILE else 2 * TILE
            assert bool(narrow) == (packed <= TILE) and q0 % tile == 0 and item_rows == min(tile, packed - q0)
            item = item0[e] + ((packed + tile - 1) // tile - 1 - q0 // tile) * hkv + g
            if shared:
                assert slot == 0 and part_row == next_part
                next_part += item_rows
                part_of.setdefault(item, []).append((part_row, item_rows))
            elif slot >= 0:
                assert slot not in slots and slot // 2 == c
                slots.add(slot)
            assert n0 == ((J + 1) // 2 if narrow else n0) and n1 == (J // 2 if narrow else n1) and 0 <= n0 <= J and 0 <= n1 <= J
            assert max(n0, n1) == J if not narrow else n0 + n1 == J
            for j in range(J):
                at, pg0, pg1, lo, hi, f0l, f0h, f1l, f1h, is_sink = tiles[11 * (m + j):11 * (m + j) + 10]
                base = at * KEYS
                assert 0 <= pg0 < pg1 <= 8 and base + 16 * pg1 <= (nk + 15) // 16 * 16
                # a page is fetched for a key that some row sees, at either end
                assert max(lo, base) < min(hi, base + KEYS) and pg0 == (max(lo, base) - base) // 16 and pg1 == (min(hi, base + KEYS) - base + 15) // 16
                for t in range(2):
                    if narrow and t != j % 2 or not narrow and j >= (n1 if t else n0):
                        continue
                    r_first = q0 + (0 if narrow else t * TILE)
                    some = np.zeros(KEYS, dtype=bool)
                    full = np.ones(KEYS, dtype=bool)
                    for r in range(r_first, min(r_first + TILE, packed)):
                        x = p + r // grp
                        # the row's own range in this tile, as the kernel forms it
                        mine_lo = max(max(0, x + 1 - window) if window else 0, all_lo)
                        if sinks and sk == 0:
                            mine_lo = 0
                        mine_hi = min(nk, x + 1) if causal else nk
                        a, b = (0, min(sk, mine_hi)) if is_sink else (max(mine_lo, sk), mine_hi)
                        a, b = max(a, base), min(b, base + KEYS)
                        keys = np.zeros(KEYS, dtype=bool)
                        if b > a:
                            keys[a - base:b - base] = True
                            met[(r0 + r // grp) * hq + g * grp + r % grp, a:b] += 1
                            assert lo <= a and b <= hi
                        some |= keys
                        full &= keys
                    fl, fh = (f1l, f1h) if t else (f0l, f0h)
                    if not narrow or t == 0:
                        says = np.zeros(KEYS, dtype=bool)
                        says[max(0, min(KEYS, fl - base)):max(0, min(KEYS, fh - base))] = True
                        assert (says == full).all(), "keys that all rows see"
    for i, (m_rows, p, nk) in enumerate(reqs):
        for r in range(m_rows):
            x, j = p + r, np.arange(longest)
            want = j < nk
            if causal:
                want &= j <= x
            if window:
                want &= (j > x - window) | (j < sinks)
            at = (int(first_row[i]) + r) * hq
            assert (met[at:at + hq] == want).all(), (i, r)
    if shared:
        assert next_part == part_rows and sorted(part_of) == list(range(items))
        for item, parts in part_of.items():
            assert firsts[item] == parts[0][0] and lasts[item] == parts[-1][0]
            for (a, m), (b, _) in zip(parts, parts[1:]):
                assert b == a + m
        for i in range(n):
            assert of[i] < n_groups
    return bool(shared)


SINKS = [
    ([(1, 299, 300)], 4, 2, 100, 4), ([(1, 0, 1), (1, 5, 6)], 4, 2, 100, 4), ([(1, 1199, 1200)], 28, 4, 256, 130), ([(5, 900, 905), (1, 1300, 1301)], 12, 2, 64, 1),
    ([(150, 300, 450)], 4, 2, 100, 20), ([(150, 0, 150)], 4, 2, 100, 20), ([(90, 1000, 1090)], 28, 4, 130, 257), ([(40, 500, 540), (0, 0, 0), (3, 700, 703)], 5, 5, 1, 1),
    ([(40, 500, 300)], 4, 2, 100, 128), ([(12, 400, 310)], 4, 2, 100, 16), ([(20, 600, 5)], 4, 2, 100, 128), ([(70, 100, 170)], 4, 2, 1000, 300), ([(300, 0, 300)], 4, 1, 17, 15),
]


@pytest.mark.parametrize("case", range(len(SINKS)))
def test_walk_with_sinks(planner, case):
    reqs, hq, hkv, window, sinks = SINKS[case]
    for sms in (152, 7, 1):
        verify(planner, reqs, hq, hkv, window=window, sinks=sinks, sms=sms)
    verify(planner, reqs, hq, hkv, causal=False, window=window, sinks=sinks)


def test_walk_with_sinks_of_random_calls(planner):
    rng = random.Random(5)
    for _ in range(60):
        hq, hkv = rng.choice(((4, 2), (7, 1), (3, 3), (16, 1)))
        reqs = []
        for _ in range(rng.randint(1, 5)):
            m, p = rng.choice((0, 1, 1, rng.randint(1, 90))), rng.choice((0, rng.randint(0, 900)))
            reqs.append((m, p, rng.choice((m + p, m + p, rng.randint(0, m + p + 40)))))
        if not any(r[0] for r in reqs):
            continue
        verify(planner, reqs, hq, hkv, causal=rng.random() < 0.8, window=rng.choice((1, 16, 128, rng.randint(1, 700))),
               sinks=rng.choice((1, 4, 128, 129, rng.randint(1, 400))), sms=rng.choice((152, 13, 2)))


PREFIXES = [
    ([(1, 900 + i, 901 + i) for i in range(8)], 4, 2, [(8, 900)], True),
    ([(1, 900 + i, 901 + i) for i in range(40)], 28, 4, [(40, 897)], True),
    ([(5, 400, 405)] * 6 + [(3, 700, 703)] * 4, 12, 2, [(6, 400), (4, 555)], True),
    ([(1, 300, 301)] * 5 + [(2, 10, 12)], 4, 2, [(5, 256), (1, 0)], True),
    ([(1, 300, 301), (0, 0, 0), (1, 350, 351), (4, 300, 304)], 4, 2, [(4, 300)], True),
    ([(0, 0, 0), (1, 1600, 1601), (1, 1700, 1701)], 7, 1, [(3, 1512)], True),
    ([(1, 600, 601), (1, 700, 701)], 7, 1, [(2, 512)], False),        # too little to earn a merge
    ([(1, 600, 601)], 7, 1, [(1, 512)], False),                       # a group of one
    ([(256, 300, 556)] * 2, 1, 1, [(2, 300)], False),                 # whole tiles of their own
    ([(1, 20, 21)] * 3, 4, 2, [(3, 0)], False),                       # nothing shared
    ([(64, 900, 964)] * 3 + [(1, 900, 901)] * 9, 4, 2, [(3, 900), (9, 900)], True),
    ([(1, 500, 500)] * 4, 4, 2, [(4, 500)], True),                    # rows without keys of their own
]


@pytest.mark.parametrize("case", range(len(PREFIXES)))
def test_walk_over_shared_prefixes(planner, case):
    reqs, hq, hkv, groups, shares = PREFIXES[case]
    for sms in (152, 11, 1):
        assert verify(planner, reqs, hq, hkv, groups=groups, sms=sms) == shares
    verify(planner, reqs, hq, hkv, groups=groups, causal=False)


def test_walk_over_shared_prefixes_of_random_calls(planner):
    rng, some = random.Random(6), 0
    for _ in range(40):
        hq, hkv = rng.choice(((4, 2), (7, 1), (3, 3), (16, 1)))
        reqs, groups = [], []
        for _ in range(rng.randint(1, 4)):
            count, shared = rng.randint(1, 7), rng.choice((0, 16, 1024, rng.randint(1, 2500)))
            groups.append((count, shared))
            for _ in range(count):
                m, extra = rng.choice((0, 1, 1, rng.randint(1, 30))), rng.choice((0, rng.randint(0, 200)))
                reqs.append((m, shared + extra, shared + extra + rng.choice((m, m, 0, rng.randint(0, m + 20)))))
        if not any(r[0] for r in reqs):
            continue
        some += verify(planner, reqs, hq, hkv, groups=groups, causal=rng.random() < 0.8, sms=rng.choice((152, 13, 2)))
    assert some > 15


# ---------------------------------------------------------------------------------------------- refusals
def test_struct_layout_matches_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    (tmp_path / "l.c").write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{HEADER}"\nint main(void){{printf("%zu %zu %zu", '
                                  "sizeof(crf_prefix), offsetof(crf_prefix, n_chunks), offsetof(crf_prefix, n_shared));return 0;}")
    subprocess.run([cc, str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [ctypes.sizeof(abi.Prefix), abi.Prefix.n_chunks.offset, abi.Prefix.n_shared.offset]


def call_sinks(lib, ctx, window=5, sinks=4, ch=((3, 5, 8, A16),), q=None, pl=None, ws=A16, ws_bytes=1 << 30, lse=None, hkv=2, d=64):  # noqa: F811
    return lib.crf_chunk_attention_sinks(ctx, ref(pl or pool()), 0, hkv, d, chunks(*ch), len(ch), ref(q or heads()), lse, 0.0, 1, window, sinks,
                                         ws, ws_bytes, None)


def call_prefix(lib, ctx, p=((2, 4),), ch=((1, 5, 6, A16), (1, 5, 6, A16)), q=None, pl=None, ws=A16, ws_bytes=1 << 30, hkv=2, d=64,  # noqa: F811
                causal=1, scale=0.0, n=None):
    arr = None if p is None else (abi.Prefix * max(1, len(p)))(*(abi.Prefix(*x) for x in p))
    return lib.crf_prefix_attention(ctx, ref(pl or pool()), 0, hkv, d, chunks(*ch), len(ch), arr, len(p or ()) if n is None else n,
                                    ref(q or heads()), None, scale, causal, ws, ws_bytes, None)


LONG = dict(ch=((1, 100000, 100001, A16),) * 4, p=((4, 99000),))


@pytest.mark.parametrize("kw,status", [
    (dict(sinks=-1), EINVAL), (dict(window=-1), EINVAL), (dict(window=0, sinks=-1), EINVAL), (dict(q=heads(x=A16 + 2)), EINVAL),
    (dict(q=heads(out=A16)), EINVAL), (dict(hkv=3), ESHAPE), (dict(d=96), EUNSUPPORTED), (dict(pl=pool(k=None)), EINVAL), (dict(lse=A16 + 2), EINVAL),
    (dict(ch=((1, 5, 6, None),)), EINVAL), (dict(ch=((1, 1 << 26, (1 << 26) + 1, A16),)), EUNSUPPORTED),
    (dict(window=40000, ch=((1, 100000, 100001, A16),), ws=A16 + 16), EINVAL), (dict(window=40000, ch=((1, 100000, 100001, A16),), ws_bytes=64), ENOMEM),
])
def test_sinks_refusals(lib, ctx, kw, status):  # noqa: F811
    assert call_sinks(lib, ctx, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(p=None, n=1), EINVAL), (dict(n=0), EINVAL), (dict(p=((1, 4), (1, 4), (1, 4))), EINVAL), (dict(p=((1, 4),)), EINVAL), (dict(p=((3, 4),)), EINVAL),
    (dict(p=((0, 4), (2, 4))), EINVAL), (dict(p=((2, -1),)), EINVAL), (dict(p=((2, 7),)), EINVAL), (dict(p=((2, 6),)), EINVAL),
    (dict(p=((1, 4), (1, 9))), EINVAL), (dict(q=heads(x_row=260)), EUNSUPPORTED), (dict(q=heads(out=A16)), EINVAL), (dict(hkv=3), ESHAPE),
    (dict(scale=-1.0), EINVAL), (dict(d=80), EUNSUPPORTED), (dict(**LONG, ws=A16 + 16), EINVAL), (dict(**LONG, ws_bytes=64), ENOMEM),
])
def test_prefix_refusals(lib, ctx, kw, status):  # noqa: F811
    assert call_prefix(lib, ctx, **kw) == status


def test_calls_without_rows_are_nothing(lib, ctx):  # noqa: F811
    assert call_sinks(lib, ctx, ch=((0, 5, 8, None),)) == abi.OK
    # what a request without rows shares is not looked at
    assert call_prefix(lib, ctx, ch=((0, 0, 0, None), (0, 3, 9, None)), p=((2, 1 << 20),)) == abi.OK


def test_workspace_sizes(lib, ctx):  # noqa: F811
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    ch = chunks(*LONG["ch"])
    p = (abi.Prefix * 1)(abi.Prefix(4, 99000))
    assert lib.crf_prefix_attention_workspace_size(ctx, 4, 2, 64, ch, 4, p, 1, 1, ref(n)) == abi.OK and n.value % 256 == 0 and n.value > 0
    assert lib.crf_prefix_attention_workspace_size(ctx, 4, 2, 64, ch, 4, p, 1, 1, None) == EINVAL
    assert lib.crf_prefix_attention_workspace_size(ctx, 4, 2, 64, ch, 4, None, 1, 1, ref(n)) == EINVAL
    assert lib.crf_prefix_attention_workspace_size(None, 4, 2, 64, ch, 4, p, 1, 1, ref(n)) == EINVAL
    assert lib.crf_chunk_attention_sinks_workspace_size(ctx, 4, 2, 64, ch, 4, 1, 50000, 4, ref(n)) == abi.OK
    assert lib.crf_chunk_attention_sinks_workspace_size(ctx, 4, 2, 64, ch, 4, 1, 50000, -1, ref(n)) == EINVAL
    # without a window, or without sinks, the call is the other one
    for window, sinks in ((0, 4), (50000, 0), (0, 0)):
        assert lib.crf_chunk_attention_sinks_workspace_size(ctx, 4, 2, 64, ch, 4, 1, window, sinks, ref(n)) == abi.OK
        assert lib.crf_chunk_attention_workspace_size(ctx, 4, 2, 64, ch, 4, 1, window, ref(m)) == abi.OK and n.value == m.value


def test_binding_of_prefixes():
    p = crf.Prefixes([3, 1], [100, 0])
    assert p.n == 2 and p.c[0].n_chunks == 3 and p.c[0].n_shared == 100 and p.c[1].n_shared == 0
    with pytest.raises(ValueError):
        crf.Prefixes([1], [1, 2])
    for bad in ([1 << 31], [-(1 << 31) - 1]):
        with pytest.raises(ValueError):
            crf.Prefixes(bad, [0])
        with pytest.raises(ValueError):
            crf.Prefixes([1], bad)
