"""Attention with sinks and over shared prefixes, against plain 64-bit formulas, with the tolerances of test_gpu_extend.py: both are
its kernel, and the join of a prefix's parts is its merge (a sum of fp32 parts, rounded once)."""
import math

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300.abi import CrfError
from tests.test_gpu_extend import BATCHES, BF16, DEV, HEADS, PAGE, Setup, gen, normal, pages_for, tables_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


class Sinks(Setup):
    def __init__(self, seed, hq, hkv, dim, chunks, window, sinks, **kw):
        self.sinks = sinks
        super().__init__(seed, hq, hkv, dim, chunks, window=window, **kw)

    def visible(self, m, p, n):
        j, at = torch.arange(n, device=DEV), torch.arange(p, p + m, device=DEV)[:, None]
        seen = torch.ones(m, n, dtype=torch.bool, device=DEV)
        if self.causal:
            seen &= j <= at
        if self.window:
            seen &= (j > at - self.window) | (j < self.sinks)
        return seen

    def run(self, ctx, scale=0.0, q=None, out=None, stream=None):
        b = self.batch()
        q = self.q if q is None else q
        out = torch.full((self.rows, self.hq, self.dim), 7.0, dtype=BF16, device=DEV) if out is None else out
        lse = torch.full((self.rows, self.hq), 7.0, device=DEV)
        ws = ctx.chunk_attention_workspace(self.pool, b, self.hq, causal=self.causal, window=self.window, sinks=self.sinks)
        ctx.chunk_attention(self.pool, 0, b, q, out, ws, lse=lse, scale=scale, causal=self.causal, window=self.window, sinks=self.sinks, stream=stream)
        return out, lse


@pytest.mark.parametrize("batch", sorted(BATCHES))
@pytest.mark.parametrize("hq,hkv,dim", HEADS)
def test_sinks_of_batches(ctx, hq, hkv, dim, batch):
    for window, sinks in ((100, 4), (33, 130)):
        s = Sinks(21, hq, hkv, dim, BATCHES[batch], window, sinks)
        s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("window", [1, 16, 100, 128, 129, 1000])
@pytest.mark.parametrize("sinks", [1, 4, 16, 127, 128, 129, 500])
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (28, 4, 128)])
def test_sinks_and_windows(ctx, hq, hkv, dim, window, sinks):
    # the last requests' rows have left their window of the cached keys behind, in part or whole
    s = Sinks(22, hq, hkv, dim, [(1, 2000), (70, 300), (300, 130), (5, 0), (12, 400, max(0, 410 - window)), (3, 700, 100)], window, sinks)
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (12, 2, 128)])
def test_sinks_without_causality(ctx, hq, hkv, dim):
    s = Sinks(23, hq, hkv, dim, [(9, 300, 500), (4, 600, 90), (90, 10, 400), (200, 700, 1100)], 64, 20, causal=False)
    s.verify(*s.run(ctx))
    ctx.check()


def test_sinks_of_long_chunks(ctx):
    s = Sinks(24, 28, 4, 128, [(1500, 5000), (1, 16000), (700, 0)], 1024, 16)
    s.verify(*s.run(ctx))
    s = Sinks(25, 4, 2, 64, [(3, 150000), (2, 40000)], 140000, 300)  # sums that start anew
    s.verify(*s.run(ctx))
    ctx.check()


def test_no_sinks_or_no_window_is_the_other_call(ctx):
    for window, sinks in ((0, 9), (70, 0)):
        s = Sinks(26, 12, 2, 128, [(40, 500), (1, 900)], window, sinks)
        out, lse = s.run(ctx)
        plain, plain_lse = Setup.run(s, ctx)
        assert torch.equal(out, plain) and torch.equal(lse, plain_lse)


def test_sinks_leave_the_pages_between_alone(ctx):
    """Table entries between the sinks and the windows may name pages that are gone, or none at all."""
    s = Sinks(27, 12, 2, 128, [(1, 5000), (20, 3000), (1, 700)], 300, 20)
    want, want_lse = s.run(ctx)
    for (m, p, n), t in zip(s.chunks, s.tables):
        hidden = ~s.visible(m, p, n).any(0)
        for page in range(pages_for(n)):
            if bool(hidden[page * PAGE:(page + 1) * PAGE].all()):
                t[page] = (-1, 2**30, -(2**31))[page % 3]
    out, lse = s.run(ctx)
    ctx.check()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_sinks_see_what_is_not_finite(ctx):
    """An infinite value of a sink and NaN in a window reach the rows that see them, and no other."""
    s = Sinks(28, 4, 2, 64, [(200, 300)], 50, 5, poison=False)
    page = s.tables[0].long()
    s.v[page[0], 0, 3, 7] = math.inf      # key 3: a sink, all rows
    s.v[page[400 // PAGE], 1, 400 % PAGE, 9] = math.nan  # key 400: rows at positions 400 .. 449
    out, _ = s.run(ctx)
    o = out.view(200, 2, 2, 64)
    assert bool(o[:, 0, :, 7].isposinf().all()) and bool(o[100:150, 1, :, 9].isnan().all())
    o[:, 0, :, 7], o[100:150, 1, :, 9] = 0, 0
    assert bool(o.isfinite().all())


# ---------------------------------------------------------------------------------------------- shared prefixes
class Shared(Setup):
    """Groups of (requests, shared keys, [(rows, own keys before them, keys behind them)]); whole shared pages in every member's
    table, the shared part of a page that the prefix ends in copied into each member's own."""

    def __init__(self, seed, hq, hkv, dim, groups, causal=True, scale_q=1.0, poison=True):
        members, self.groups = [], []
        for n, rows in groups:
            self.groups.append((len(rows), n))
            members += [(m, n + before, n + before + m + behind) for m, before, behind in rows]
        super().__init__(seed, hq, hkv, dim, members, causal=causal, scale_q=scale_q, poison=poison)
        at = 0
        for count, n in self.groups:
            # the first with rows (of the others the pages of Setup hold no numbers)
            lead = next(t for t, c in zip(self.tables[at:at + count], self.chunks[at:at + count]) if c[0] > 0)
            whole = n // PAGE
            for t in self.tables[at:at + count]:
                if n % PAGE and t is not lead and len(t) > whole:
                    a, b = lead[whole].long(), t[whole].long()
                    self.k[b, :, :n % PAGE], self.v[b, :, :n % PAGE] = self.k[a, :, :n % PAGE], self.v[a, :, :n % PAGE]
                t[:whole] = lead[:whole]
            at += count

    def prefixes(self):
        return crf.Prefixes([g[0] for g in self.groups], [g[1] for g in self.groups])

    def run(self, ctx, scale=0.0, q=None, out=None, stream=None, with_lse=True):
        b, p = self.batch(), self.prefixes()
        q = self.q if q is None else q
        out = torch.full((self.rows, self.hq, self.dim), 7.0, dtype=BF16, device=DEV) if out is None else out
        lse = torch.full((self.rows, self.hq), 7.0, device=DEV) if with_lse else None
        ws = ctx.prefix_attention_workspace(self.pool, b, p, self.hq, causal=self.causal)
        ctx.prefix_attention(self.pool, 0, b, p, q, out, ws, lse=lse, scale=scale, causal=self.causal, stream=stream)
        return out, lse


# Groups are shared where that saves enough: all but those of the last three.
GROUPS = {
    "samples": [(9000, [(1, i, 0) for i in range(30)])],
    "many samples": [(4096, [(1, 3 * i, 0) for i in range(100)])],
    "drafts": [(7001, [(5, 0, 0)] * 40 + [(3, 40, 0)])],
    "groups and one alone": [(3700, [(2, 9, 0)] * 50), (0, [(3, 20, 0)]), (4607, [(1, 0, 0), (4, 130, 0), (1, 500, 0)] * 10)],
    "ends of pages and tiles": [(4096, [(1, 0, 0)] * 30), (4095, [(1, 0, 0)] * 30), (4097, [(1, 0, 0)] * 30), (4080, [(1, 16, 0)] * 30)],
    "long rows": [(5100, [(40, 0, 0), (1, 5, 0), (70, 20, 0), (9, 0, 0)] * 12)],
    "requests without rows": [(8000, [(0, 0, 0), (1, 4, 0), (0, 5, 0), (1, 7, 0), (3, 0, 0), (1, 0, 0), (0, 9, 0)] * 9)],
    "no keys of their own": [(6000, [(1, 0, -1)] * 50 + [(2, 3, -5)] * 3)],
    "keys behind the rows": [(6000, [(1, 0, 30)] * 50 + [(2, 3, 200)] * 3)],
    # requests whose own keys are long: split from the shared ones where heads are many, beside a folded group and one alone
    "long keys of their own": [(6000, [(1, 1500 + 16 * i, 0) for i in range(24)]), (5000, [(2, 3, 0)] * 30), (0, [(1, 40, 0)])],
    "rows of several tiles": [(6000, [(13, 7 * i, 0) for i in range(70)])],
    "few samples": [(900, [(1, i, 0) for i in range(8)])],
    "two groups": [(700, [(2, 9, 0)] * 5), (0, [(3, 20, 0)]), (1607, [(1, 0, 0), (4, 130, 0), (1, 500, 0)])],
    "short": [(17, [(1, 0, 0)] * 3), (3, [(1, 1, 0)])],
}


def shared_kernel(ctx, call):
    """Whether the call ran the kernel of shared prefixes."""
    ctx.profile_enable(True)
    try:
        call()
        torch.cuda.synchronize()
        return "prefix_attention" in ctx.profile_read()
    finally:
        ctx.profile_enable(False)


def test_which_groups_are_shared(ctx):
    unshared = {"few samples", "two groups", "short"}
    for hq, hkv, dim in HEADS[:3]:
        for name in sorted(GROUPS):
            s = Shared(30, hq, hkv, dim, GROUPS[name], poison=False)
            assert shared_kernel(ctx, lambda: s.run(ctx)) == (name not in unshared), (name, hq)  # noqa: B023


@pytest.mark.parametrize("name", sorted(GROUPS))
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (28, 4, 128), (16, 1, 128)])
def test_shared_prefixes(ctx, hq, hkv, dim, name):
    s = Shared(31, hq, hkv, dim, GROUPS[name])
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (28, 4, 128)])
def test_shared_prefixes_without_causality(ctx, hq, hkv, dim):
    s = Shared(32, hq, hkv, dim, [(4200, [(3, 0, 40), (1, 0, 0), (2, 7, 1), (1, 100, 0)] * 12), (40, [(90, 0, 0)])], causal=False)
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("scale_q", [0.0, 8.0, 60.0])
def test_shared_prefixes_of_sharp_and_flat_scores(ctx, scale_q):
    s = Shared(33, 12, 2, 128, [(8500, [(2, 10, 0)] * 30)], scale_q=scale_q)
    s.verify(*s.run(ctx))


def test_shared_prefix_of_most_requests(ctx):
    s = Shared(34, 4, 2, 64, [(4600, [(1, i, 0) for i in range(crf.abi.MAX_CHUNKS)])])
    s.verify(*s.run(ctx))
    s = Shared(35, 4, 2, 64, [(7000, [(1, 5, 0), (2, 9, 0)])] * 64)
    s.verify(*s.run(ctx))
    ctx.check()


def test_long_shared_prefix(ctx):
    s = Shared(36, 28, 4, 128, [(20000, [(1, i, 0) for i in range(32)])])
    s.verify(*s.run(ctx))
    s = Shared(37, 2, 1, 64, [(200000, [(1, 5, 0), (3, 50, 0)] * 6)])
    s.verify(*s.run(ctx))
    ctx.check()


def test_shared_prefix_strides_and_outputs(ctx):
    s = Shared(38, 12, 2, 128, [(9000, [(2, 5, 0)] * 25)])
    want, lse = s.run(ctx)
    wide = torch.full((s.rows + 2, 14, 136), 3.0, dtype=BF16, device=DEV)
    q = torch.zeros(12, s.rows, 128, dtype=BF16, device=DEV).copy_(s.q.transpose(0, 1)).transpose(0, 1)
    keep = wide.clone()
    view = wide[1:-1, 1:13, :128]
    got, none = s.run(ctx, q=q, out=view, with_lse=False)
    assert none is None and torch.equal(got, want)
    view.copy_(keep[1:-1, 1:13, :128])
    assert torch.equal(wide, keep)  # rows behind the last sequence, and everything else outside the view


def test_shared_prefix_of_bad_pages(ctx):
    s = Shared(39, 4, 2, 64, [(9000, [(1, 5, 0)] * 60)], poison=False)
    s.tables[0][3], s.tables[4][562] = len(s.k), -1
    s.run(ctx)
    with pytest.raises(CrfError, match="EINVAL"):
        ctx.check()
    ctx.check()


def test_shared_prefix_sees_what_is_not_finite(ctx):
    s = Shared(40, 4, 2, 64, [(9000, [(1, 5, 0)] * 60)], poison=False)
    s.v[s.tables[0][10].long(), 0, 4, 7] = math.inf     # shared: all rows
    s.v[s.tables[2][9003 // PAGE].long(), 1, 9003 % PAGE, 9] = math.nan  # request 2's own
    out, _ = s.run(ctx)
    o = out.view(60, 2, 2, 64)
    assert bool(o[:, 0, :, 7].isposinf().all()) and bool(o[2, 1, :, 9].isnan().all())
    o[:, 0, :, 7], o[2, 1, :, 9] = 0, 0
    assert bool(o.isfinite().all())


@pytest.mark.parametrize("kind", ["sinks", "prefix"])
def test_calls_repeat_their_bits_on_streams_and_in_graphs(ctx, kind):
    if kind == "sinks":
        s = Sinks(41, 28, 4, 128, [(1, 5000), (60, 3000), (1, 9000)], 700, 9)
        b = s.batch()
        ws = lambda: ctx.chunk_attention_workspace(s.pool, b, 28, window=700, sinks=9)  # noqa: E731
        call = lambda o, l, w, **kw: ctx.chunk_attention(s.pool, 0, b, s.q, o, w, lse=l, window=700, sinks=9, **kw)  # noqa: E731
    else:
        s = Shared(42, 28, 4, 128, [(9000, [(1, 7 * i, 0) for i in range(16)])])
        b, p = s.batch(), s.prefixes()
        ws = lambda: ctx.prefix_attention_workspace(s.pool, b, p, 28)  # noqa: E731
        call = lambda o, l, w, **kw: ctx.prefix_attention(s.pool, 0, b, p, s.q, o, w, lse=l, **kw)  # noqa: E731
    new = lambda: (torch.zeros_like(s.q), torch.zeros(s.q.shape[:2], device=DEV), ws().fill_(255))  # noqa: E731
    first, second, third = new(), new(), new()
    call(*first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(*second, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*third)
    for _ in range(3):
        third[0].zero_(), third[1].zero_(), third[2].fill_(255)
        graph.replay()
    torch.cuda.synchronize()
    for a, c, d in zip(first[:2], second, third):
        assert torch.equal(a, c) and torch.equal(a, d)
    ctx.check()


def test_a_fork_is_continued_and_scored(ctx):
    """What the calls are for, in a row: a cached prefix forks, every fork's next rows are normed, turned and appended, attended over the
    shared prefix, attended again through a window with sinks, and the logits of an output head scored."""
    g = gen(43)
    hq, hkv, dim, n, forks, m = 12, 2, 128, 6005, 30, 3
    (lead,), total = tables_of(g, [pages_for(n + m)], spare=60)
    kp, vp = normal(g, total, hkv, PAGE, dim), normal(g, total, hkv, PAGE, dim)
    pool = crf.KVPool([kp], [vp])
    refs = torch.zeros(total, dtype=torch.int32, device=DEV)
    refs[lead[:pages_for(n)].long()] = 1
    tables = [torch.zeros(pages_for(n + m), dtype=torch.int32, device=DEV) for _ in range(forks)]
    whole = crf.PageTables([lead] * forks, [n] * forks, tables)
    ctx.pages_fork(pool, refs, whole, ctx.pages_workspace(total, whole))
    ctx.check()
    # room for the new rows: n + m tokens fill no page that n does not
    assert pages_for(n + m) == pages_for(n)
    qkv = normal(g, forks * m, hq + 2 * hkv, dim)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    gain, rope = (1 + 0.1 * normal(g, dim, dtype=torch.float32)).to(BF16), crf.Rope(dim, theta=1e6)
    chunks = crf.Chunks(tables, [m] * forks, [n] * forks)
    turned = torch.empty(forks * m, hq, dim, dtype=BF16, device=DEV)
    ctx.cache_append(pool, 0, chunks, k, v, q=q, q_out=turned, rope=rope, q_gain=gain, k_gain=gain)
    prefixes = crf.Prefixes([forks], [n])
    o, lse = torch.empty_like(turned), torch.empty(forks * m, hq, device=DEV)
    ctx.prefix_attention(pool, 0, chunks, prefixes, turned, o, ctx.prefix_attention_workspace(pool, chunks, prefixes, hq), lse=lse)
    near, near_lse = torch.empty_like(turned), torch.empty(forks * m, hq, device=DEV)
    ctx.chunk_attention(pool, 0, chunks, turned, near, ctx.chunk_attention_workspace(pool, chunks, hq, window=200, sinks=4), lse=near_lse, window=200, sinks=4)
    head = normal(g, hq * dim, 1000) * 0.02
    logits = (o.reshape(forks * m, -1).float() @ head.float())
    targets = torch.randint(0, 1000, (forks * m,), device=DEV, generator=g, dtype=torch.int32)
    lp, ids = torch.empty(forks * m, device=DEV), torch.empty(forks * m, 4, dtype=torch.int32, device=DEV)
    ctx.logprobs(logits, targets, logprob=lp, top_ids=ids)
    ctx.check()
    # the same, each request by itself, in 64 bits from what the pages hold now
    s = Setup.__new__(Setup)
    s.hq, s.hkv, s.dim, s.causal, s.window, s.rows = hq, hkv, dim, True, 0, forks * m
    s.chunks, s.tables, s.k, s.v, s.q = [(m, n, n + m)] * forks, tables, kp, vp, turned
    s.verify(o, lse)
    w = Sinks.__new__(Sinks)
    w.__dict__.update(s.__dict__, window=200, sinks=4)
    w.verify(near, near_lse)
    # each fork's page that the prefix ends in is its own and holds its own new keys
    assert len({int(t[n // PAGE]) for t in tables}) == forks
    want = torch.log_softmax(logits.double(), 1).gather(1, targets.long()[:, None])[:, 0]
    assert bool(((lp.double() - want).abs() <= 2.0**-15 * (1 + want.abs())).all())
    assert torch.equal(ids.long(), torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :4])
