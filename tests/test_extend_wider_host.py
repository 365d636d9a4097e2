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
#include "prefix_attn.cu"
namespace crf {  // what the launches need and the plan does not
PdlScope::PdlScope() : prev_(false) {}
PdlScope::~PdlScope() {}
bool pdl_active() { return false; }
}  // namespace crf
using namespace crf;
static ChunkArgs<kPrefix> args;
static ChunkArgs<kSinks> with_sinks;
static AttnPlan plan;
static PrefixGroups groups;
static bool prefixes;
// The plan of requests whose page tables are rows of `tables`. info: shared, entries, split groups, items, part rows, cuts, whether any group shares;
// returns the number of CTAs. Whether a group is worth sharing is decided for `sharers` SMs.
extern "C" int make(int n, const int* n_new, const int* pos, const int* n_keys, const int* tables, int stride, int n_groups, const int* count,
                    const int* keys, int hq, int hkv, int causal, int window, int sinks, int sms, int sharers, int* info, int* firsts, int* lasts) {
  ChunkTable t = {};
  t.n = n;
  for (int i = 0; i < n; ++i) t.row0[i + 1] = t.row0[i] + n_new[i], t.pos[i] = pos[i], t.n_keys[i] = n_keys[i], t.pt[i] = tables + i * stride;
  for (int i = n; i < kMaxChunks; ++i) t.row0[i + 1] = t.row0[n];
  prefixes = n_groups > 0;
  if (!prefixes) {
    memset(&with_sinks, 0, sizeof(with_sinks));
    with_sinks.c = SinksTable{t, sinks};
    plan_runs<kSinksCosts>(with_sinks.c, hq, hkv, causal != 0, window, sms, nullptr, &plan.runs);
    memcpy(with_sinks.run, plan.runs.run, sizeof(with_sinks.run));
    with_sinks.d.n_q_heads = hq, with_sinks.d.n_kv_heads = hkv, with_sinks.d.causal = causal != 0, with_sinks.d.window = window;
    const int v[7] = {0, n, 0, 0, 0, plan.runs.cuts, 0};
    memcpy(info, v, sizeof(v));
    return plan.runs.ctas;
  }
  memset(&args, 0, sizeof(args));
  memset(&groups, 0, sizeof(groups));
  AttnTable& a = args.c;
  share_prefixes(t, count, keys, n_groups, hq, hkv, causal != 0, sharers, &a, &groups);
  plan_prefix_attention(a, groups.groups > 0, hq, hkv, causal != 0, sms, &plan);
  memcpy(args.run, plan.runs.run, sizeof(args.run));
  args.d.n_q_heads = hq, args.d.n_kv_heads = hkv, args.d.causal = causal != 0, args.d.window = 0;
  args.prefix.on = plan.shared;
  args.prefix.first = firsts, args.prefix.last = lasts;
  memcpy(args.prefix.item0, plan.item0, sizeof(plan.item0));
  int row = 0;
  for (int b = 0; b < plan.runs.ctas; ++b) args.prefix.row0[b] = row, row += static_cast<int>(plan.run_rows[b]);
  const int v[7] = {plan.shared, a.n, groups.groups, plan.items, static_cast<int>(plan.part_rows), plan.runs.cuts, groups.any};
  memcpy(info, v, sizeof(v));
  return plan.runs.ctas;
}
extern "C" void table(int* row0, int* rows, int* item0, int* of) {
  if (!prefixes)
    for (int i = 0; i < with_sinks.c.n; ++i) row0[i] = with_sinks.c.row0[i], rows[i] = rows_of(with_sinks.c, i), item0[i] = 0, of[i] = -1;
  else
    for (int i = 0; i < args.c.n; ++i) row0[i] = args.c.row0[i], rows[i] = args.c.rows[i], item0[i] = plan.item0[i], of[i] = i < groups.groups ? -2 : groups.of[i - groups.groups];
}
static int page_at(const ChunkArgs<kSinks>&, const SegmentOf<kSinks>& s, int j, int p) { return s.pt[cache_tile(s, j) * kPagesPerTile + p]; }
static int page_at(const ChunkArgs<kPrefix>& a, const SegmentOf<kPrefix>& s, int j, int p) {
  int member = -1;
  for (int i = 0; i < a.c.members[s.entry]; ++i) member += a.c.m_page0[a.c.member0[s.entry] + i] <= (cache_tile(s, j) - s.ns) * 8 + p;
  return page_of(a.c, s, j, p, member);
}
// A CTA's segments, 12 numbers each; their tiles, 16 each: the range of what all rows of the two chains see, first and last page, the pages; and what
// each row sees of each tile, 2 each. Returns the segments.
template <int FORM>
static int walk_form(const ChunkArgs<FORM>& a, int part_row, int cta, int* seg, int* tiles, int max_tiles, int* ranges, int max_ranges) {
  Walk<FORM> w;
  w.at = a.run[cta];
  w.part_row = part_row;
  int n = 0, m = 0, r = 0;
  const int grp = a.d.n_q_heads / a.d.n_kv_heads;
  for (;; ++n) {
    SegmentOf<FORM> s;
    w.next(a, cta, s);
    if (s.end) return n;
    const int v[12] = {s.g, s.q0, s.rows, s.entry, s.narrow, s.slot, s.J, s.n0, s.n1, s.part_row, s.item_rows, m};
    memcpy(seg + 12 * n, v, sizeof(v));
    const PageSpan<FORM> pages(s);
    for (int j = 0; j < s.J; ++j, ++m) {
      if (m >= max_tiles) return -1;
      const int k0 = cache_tile(s, j) * kN;
      const KeyRange f0 = range_in(s, j, s.full0), f1 = range_in(s, j, s.full1), all = range_in(s, j, KeyRange{s.all_lo, s.all_hi});
      int* t = tiles + 16 * m;
      t[0] = f0.lo - k0, t[1] = f0.hi - k0, t[2] = f1.lo - k0, t[3] = f1.hi - k0, t[4] = pages.first(j), t[5] = pages.last(j), t[6] = all.lo - k0, t[7] = all.hi - k0;
      for (int p = 0; p < 8; ++p) t[8 + p] = p >= t[4] && p < t[5] ? page_at(a, s, j, p) : -1;
      for (int q = s.q0; q < s.q0 + s.item_rows; ++q, ++r) {
        if (r >= max_ranges) return -2;
        const KeyRange k = range_in(s, j, row_keys(a.c, s, q / grp, a.d.causal, a.d.window));
        ranges[2 * r] = k.lo - k0, ranges[2 * r + 1] = k.hi - k0;
      }
    }
  }
}
extern "C" int walk(int cta, int* seg, int* tiles, int max_tiles, int* ranges, int max_ranges) {
  return prefixes ? walk_form(args, args.prefix.row0[cta], cta, seg, tiles, max_tiles, ranges, max_ranges)
                  : walk_form(with_sinks, 0, cta, seg, tiles, max_tiles, ranges, max_ranges);
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


def verify(so, reqs, hq, hkv, causal=True, window=0, sinks=0, groups=(), sms=152, sharers=0):
    """reqs: (rows, position, keys); groups: (requests, shared keys). Whether the call shares anything, and how many of its groups are split."""
    n, grp = len(reqs), hq // hkv
    longest = max(r[2] for r in reqs)
    pages = (longest + 15) // 16
    tables = np.arange(n * max(1, pages), dtype=np.int32).reshape(n, -1)  # page p of request i: i pages + p
    shared_of = [k for c, k in groups for _ in range(c)] or [0] * n
    group_of = [g for g, (c, _) in enumerate(groups) for _ in range(c)] or list(range(n))
    info = (ctypes.c_int * 7)()
    firsts, lasts = (ctypes.c_int * 100000)(*[-1] * 100000), (ctypes.c_int * 100000)(*[-1] * 100000)
    ctas = so.make(n, ints([r[0] for r in reqs]), ints([r[1] for r in reqs]), ints([r[2] for r in reqs]), tables.ctypes.data_as(ctypes.c_void_p),
                   tables.shape[1], len(groups), ints([g[0] for g in groups]), ints([g[1] for g in groups]), hq, hkv, int(causal), window, sinks, sms,
                   sharers, info, firsts, lasts)
    shared, entries, split, items, part_rows, cuts, any_shares = info
    assert 0 < ctas <= sms and cuts <= 256 and bool(shared) == (split > 0)
    tab = [(ctypes.c_int * entries)() for _ in range(4)]
    so.table(*tab)
    row0, rows, item0, of = ([int(x) for x in t] for t in tab)
    request = np.repeat(np.arange(n), [r[0] for r in reqs])  # of each row
    first_row = np.cumsum([0] + [r[0] for r in reqs])
    met = np.zeros((len(request) * hq, longest), dtype=np.int32)
    part_of = {}  # item -> [(part row, rows)], in order of runs
    seg, tiles, ranges = (ctypes.c_int * (12 * 4000))(), np.zeros((60000, 16), dtype=np.int32), np.zeros((3000000, 2), dtype=np.int32)
    slots, next_part = set(), 0
    for c in range(ctas):
        count = so.walk(c, seg, tiles.ctypes.data_as(ctypes.c_void_p), len(tiles), ranges.ctypes.data_as(ctypes.c_void_p), len(ranges))
        assert 0 <= count < 4000
        at = 0
        for k in range(count):
            g, q0, packed, e, narrow, slot, J, n0, n1, part_row, item_rows, m = seg[12 * k:12 * k + 12]
            tile = TILE if packed <= TILE else 2 * TILE
            assert packed == rows[e] * grp and bool(narrow) == (packed <= TILE) and q0 % tile == 0 and item_rows == min(tile, packed - q0)
            item = item0[e] + ((packed + tile - 1) // tile - 1 - q0 // tile) * hkv + g
            if shared:
                assert slot == 0 and part_row == next_part
                next_part += item_rows
                part_of.setdefault(item, []).append((part_row, item_rows))
            elif slot >= 0:
                assert slot not in slots and slot // 2 == c
                slots.add(slot)
            assert 0 <= n0 <= J and 0 <= n1 <= J and (n0 + n1 == J and 0 <= n0 - n1 <= 1 if narrow else max(n0, n1) == J)
            # a chain gives back the K/V tiles that it does not go through at the segment's end: more than two of them are
            # more than the ring's five slots, which the other chain would wait for without end
            assert narrow or min(n0, n1) == 0 or J - min(n0, n1) <= 2
            for j in range(J):
                t, mine = tiles[m + j], ranges[at:at + item_rows]
                at += item_rows
                pg0, pg1 = t[4:6]
                assert 0 <= pg0 < pg1 <= 8
                lo, hi = max(0, t[6]), min(KEYS, t[7])
                assert lo < hi and pg0 == lo // 16 and pg1 == (hi + 15) // 16  # a page is fetched for what some row sees, at either end
                a, b = np.clip(mine[:, 0], 0, KEYS), np.clip(mine[:, 1], 0, KEYS)
                x = np.arange(KEYS)
                sees = (x >= a[:, None]) & (x < b[:, None])
                assert (~sees.any(1) | ((a >= lo) & (b <= hi))).all()
                for ch in range(2):
                    part = sees if narrow else sees[ch * TILE:(ch + 1) * TILE]
                    if not len(part) or narrow and ch != j % 2:
                        continue
                    if not narrow and j >= (n1 if ch else n0):
                        assert not part.any()  # the chain does not go through this tile
                        continue
                    says = np.zeros(KEYS, dtype=bool)
                    says[max(0, min(KEYS, t[2 * ch])):max(0, min(KEYS, t[2 * ch + 1]))] = True
                    exact = part.all(0)
                    # of requests side by side the bound may leave out what all see by chance
                    assert (says <= exact).all() and (says.all() or of[e] == -1 and groups or (says == exact).all()), "keys that all rows see"
                if not sees.any():
                    continue
                ids = np.where(np.arange(8) >= 0, t[8:16], -1)
                req_of_page, page = ids // tables.shape[1], ids % tables.shape[1]
                q, y = np.nonzero(sees)
                p = y // 16
                assert (p >= pg0).all() and (p < pg1).all()
                row = row0[e] + (q0 + q) // grp
                key = page[p] * 16 + y % 16
                i, whose = request[row], req_of_page[p]
                # a page of the row's own request, or a shared key of another of its group's
                assert ((whose == i) | (np.array(group_of)[whose] == np.array(group_of)[i]) & (key < np.array(shared_of)[i])).all()
                assert (key < np.array([r[2] for r in reqs])[i]).all()
                np.add.at(met, (row * hq + g * grp + (q0 + q) % grp, key), 1)
    j = np.arange(longest)
    for i, (m_rows, p, nk) in enumerate(reqs):
        for r in range(m_rows):
            x = p + r
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
    # every row is one entry's, beside a split group's
    own = sorted((row0[e], rows[e]) for e in range(entries) if of[e] != -2 and rows[e])
    assert sum(r for _, r in own) == len(request) and all(a + r == b for (a, r), (b, _) in zip(own, own[1:]))
    return bool(any_shares), split


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


PREFIXES = [  # requests, heads, groups, how many groups are split; None: nothing is shared
    ([(1, 900 + i, 901 + i) for i in range(8)], 4, 2, [(8, 900)], 0),
    ([(1, 900 + i, 901 + i) for i in range(40)], 28, 4, [(40, 897)], 0),
    ([(5, 400, 405)] * 6 + [(3, 700, 703)] * 4, 12, 2, [(6, 400), (4, 555)], 0),
    ([(1, 300, 301)] * 5 + [(2, 10, 12)], 4, 2, [(5, 256), (1, 0)], 0),
    ([(1, 300, 301), (0, 0, 0), (1, 350, 351), (4, 300, 304)], 4, 2, [(4, 300)], 0),
    ([(0, 0, 0), (1, 1600, 1601), (1, 1700, 1701)], 7, 1, [(3, 1512)], 0),
    ([(1, 600, 601)], 7, 1, [(1, 512)], None),                       # a group of one
    ([(256, 300, 556)] * 2, 1, 1, [(2, 300)], None),                 # whole tiles of their own
    ([(1, 20, 21)] * 3, 4, 2, [(3, 0)], None),                       # nothing shared
    ([(64, 900, 964)] * 3 + [(1, 900, 901)] * 9, 4, 2, [(3, 900), (9, 900)], 0),
    ([(1, 500, 500)] * 4, 4, 2, [(4, 500)], 0),                      # rows without keys of their own
    ([(1, 900 + 500 * i, 901 + 500 * i) for i in range(5)], 4, 2, [(5, 900)], 0),
    ([(1, 6000 + 30 * i, 6001 + 30 * i) for i in range(24)], 28, 4, [(24, 4000)], 1),   # long keys of their own: split
    ([(1, 5000, 5001)] * 24 + [(1, 3000, 3001)] * 6, 28, 4, [(24, 3000), (6, 3000)], 1),
    ([(1, 3000, 3001)] * 6 + [(1, 5000, 5001)] * 24 + [(1, 60, 61)], 28, 4, [(6, 3000), (24, 3000), (1, 0)], 1),
    ([(13, 1900, 1913)] * 12 + [(13, 1900, 1940)], 28, 4, [(13, 1900)], 0),                 # several tiles of rows
    ([(3, 1900, 5000)] * 4 + [(3, 1900, 8000)] * 3, 28, 4, [(7, 1900)], 0),                 # keys behind the rows
]


@pytest.mark.parametrize("case", range(len(PREFIXES)))
def test_walk_over_shared_prefixes(planner, case):
    reqs, hq, hkv, groups, split = PREFIXES[case]
    for sms in (152, 11, 1):
        got = verify(planner, reqs, hq, hkv, groups=groups, sms=sms)
        assert got == (split is not None, split or 0)
    verify(planner, reqs, hq, hkv, groups=groups, causal=False)


def test_little_work_is_not_shared(planner):
    # 24 units an SM have to be saved, 40 where a group is split
    for requests, keys, shares in ((32, 1000, False), (8, 15000, True), (32, 15000, True), (2, 15000, False)):
        reqs = [(1, keys + 5, keys + 6)] * requests
        assert verify(planner, reqs, 28, 4, groups=[(requests, keys)], sharers=152)[0] == shares


def test_walk_over_shared_prefixes_of_random_calls(planner):
    rng, some, splits = random.Random(6), 0, 0
    for _ in range(40):
        hq, hkv = rng.choice(((4, 2), (7, 1), (3, 3), (16, 1)))
        reqs, groups = [], []
        for _ in range(rng.randint(1, 4)):
            count, shared, far = rng.randint(1, 7), rng.choice((0, 16, 1024, rng.randint(1, 2500))), rng.choice((200, 4000))
            groups.append((count, shared))
            for _ in range(count):
                m, extra = rng.choice((0, 1, 1, rng.randint(1, 30))), rng.choice((0, rng.randint(0, far)))
                reqs.append((m, shared + extra, shared + extra + rng.choice((m, m, 0, rng.randint(0, m + 20)))))
        if not any(r[0] for r in reqs):
            continue
        got = verify(planner, reqs, hq, hkv, groups=groups, causal=rng.random() < 0.8, sms=rng.choice((152, 13, 2)))
        some, splits = some + got[0], splits + (got[1] > 0)
    assert some > 15 and splits > 0


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
