"""Calls that extend a recovered cache with new tokens, against plain 64-bit formulas.

Tolerances count roundings. Rotary: half a step of the type relative to the value (finfo.eps / 2), and 2^-21
(|x| + |y|) magnitude for the fp32 arithmetic (angle in fp32 2^-24 pi/4, sine and cosine one unit in the last place,
four roundings: under 4e-7). Attention: weights enter the product with v rounded to bf16 (2^-8 of each weight
at most) and o is rounded to bf16 (2^-8 of the value); fp32 sums, maxima and exponentials add 2^-12 of
sum w |v|. lse: each fp32 score is off by at most 2^-16 scale sum |q k| (128 products summed in fp32), its
exponential and the sum by 2^-17. Copies, counts and tables are exact."""
import math

import numpy as np
import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300.abi import CrfError

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, PAGE = torch.bfloat16, 16


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def tables_of(g, counts, spare=3):
    """Page tables dealt from a random permutation of the pool, and the pool's size."""
    perm = torch.randperm(sum(counts) + spare, device=DEV, generator=g).to(torch.int32)
    return [t.contiguous() for t in perm[: sum(counts)].split(list(counts))], len(perm)


def pages_for(n):
    return (n + PAGE - 1) // PAGE


# ---------------------------------------------------------------------------------------------- rotary
ROPES = {
    "whole": dict(theta=1e4), "part": dict(theta=1e6, rot_dim=32), "linear": dict(theta=1e4, scaling="linear", factor=8.0),
    "base": dict(theta=5e5, scaling="base", factor=4.0),
    "bands": dict(theta=1e6, scaling="bands", factor=4.0, low=1.0, high=32.0, original=8192, magnitude=1.1386),
}


def frequencies(dim, a):
    rot, s = a.get("rot_dim", dim), a.get("factor", 1.0)
    theta = a["theta"] * (s ** (rot / (rot - 2)) if a.get("scaling") == "base" else 1.0)
    f = np.power(theta, -np.arange(0, rot, 2, dtype=np.float64) / rot)
    if a.get("scaling") == "linear":
        f = f / s
    if a.get("scaling") == "bands":
        g = np.clip((a["original"] * f / (2 * np.pi) - a["low"]) / (a["high"] - a["low"]), 0, 1)
        f = f * (g + (1 - g) / s)
    return torch.tensor(f, device=DEV)


def rotate64(x, pos, dim, a, inverse=False):
    """(rotated, |x| + |y| of each element's pair, zero where nothing turns) in 64 bits."""
    rot, x = a.get("rot_dim", dim), x.double()
    ang = pos.double()[:, None] * frequencies(dim, a)[None]
    c, s = ang.cos()[:, None], ang.sin()[:, None] * (-1 if inverse else 1)
    i0, i1 = (torch.arange(rot // 2), torch.arange(rot // 2, rot)) if a.get("layout", "half") == "half" else \
        (torch.arange(0, rot, 2), torch.arange(1, rot, 2))
    y, size, m = x.clone(), torch.zeros_like(x), a.get("magnitude", 1.0)
    u, v = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = m * (u * c - v * s), m * (v * c + u * s)
    size[..., i0] = size[..., i1] = abs(m) * (u.abs() + v.abs())
    return y, size


def assert_rotated(got, x, pos, dim, a, inverse=False):
    want, size = rotate64(x, pos, dim, a, inverse)
    # below the smallest normal number (fp16: 2^-14) a type's steps stay those of that number
    t = torch.finfo(got.dtype)
    tol = t.eps / 2 * want.abs().clamp(min=t.tiny) * 1.001 + 2.0**-21 * size
    worst = float(((got.double() - want).abs() - tol).max())
    assert worst <= 0, worst


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("name", sorted(ROPES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_rotary_of_types_layouts_and_scalings(ctx, dtype, name, layout):
    a = dict(ROPES[name], layout=layout)
    g = gen(1)
    for rows, hq, hk, dim in ((1, 4, 2, 64), (37, 28, 4, 128), (300, 3, 1, 64)):
        x = normal(g, rows, hq + hk, dim, dtype=dtype)
        pos = torch.randint(0, 131072, (rows,), device=DEV, generator=g, dtype=torch.int32)
        q, k = torch.empty(rows, hq, dim, dtype=dtype, device=DEV), torch.empty(rows, hk, dim, dtype=dtype, device=DEV)
        for inverse in (False, True):
            ctx.rotary(crf.Rope(dim, **a), pos, x[:, :hq], q, k=x[:, hq:], k_out=k, inverse=inverse)
            assert_rotated(q, x[:, :hq], pos, dim, a, inverse)
            assert_rotated(k, x[:, hq:], pos, dim, a, inverse)
    ctx.check()


@pytest.mark.parametrize("dim,rot", [(2, 2), (6, 4), (80, 40), (96, 96), (256, 256), (256, 2), (66, 66), (64, 20)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_of_odd_heads(ctx, dim, rot, layout):
    g = gen(2)
    a = dict(theta=1e4, rot_dim=rot, layout=layout)
    x = normal(g, 19, 5, dim)
    pos = torch.randint(0, 5000, (19,), device=DEV, generator=g, dtype=torch.int32)
    out = torch.empty_like(x)
    ctx.rotary(crf.Rope(dim, **a), pos, x, out)
    assert_rotated(out, x, pos, dim, a)


def test_rotary_strides_alignment_and_in_place(ctx):
    g = gen(3)
    a = dict(theta=1e4)
    big = normal(g, 11, 9, 72)
    for view in (big[:, 2:7, 3:67], big[:, :, 8:72], big.transpose(0, 1)[..., :64]):
        pos = ints(*range(100, 100 + len(view)))
        keep = big.clone()
        want = view.clone()
        ctx.rotary(crf.Rope(64, **a), pos, view)  # in place, whatever the strides and the alignment
        assert_rotated(view, want, pos, 64, a)
        view.copy_(want)
        assert torch.equal(big, keep)  # nothing outside the view was touched
    # heads outside, rows inside
    x = normal(g, 4, 13, 64).transpose(0, 1)
    out = torch.empty(4, 13, 64, dtype=BF16, device=DEV).transpose(0, 1)
    pos = ints(*range(13))
    ctx.rotary(crf.Rope(64, **a), pos, x, out)
    assert_rotated(out, x, pos, 64, a)


def test_rotary_positions_far_negative_and_none(ctx):
    g = gen(4)
    a = dict(theta=1e6)
    pos = ints(0, -1, -70000, 2**31 - 1, -(2**31), 1 << 24, 12345678)
    x = normal(g, 7, 2, 128, dtype=torch.float32)
    out = torch.empty_like(x)
    ctx.rotary(crf.Rope(128, **a), pos, x, out)
    # the frequency itself is a rounded number: 2^31 positions carry its 2^-53 to 2^-21
    want, size = rotate64(x, pos, 128, a)
    assert bool(((out.double() - want).abs() <= 2.0**-24 * want.abs() + 2.0**-20 * size).all())
    assert torch.equal(out[0], x[0])
    ctx.rotary(crf.Rope(128, **a), pos[:0], x[:0], out[:0])
    ctx.check()


def test_rotary_inverse_is_the_gradient(ctx):
    g = gen(5)
    a = dict(theta=1e4, rot_dim=32, scaling="bands", factor=4.0, low=1.0, high=16.0, original=512, magnitude=1.2)
    x, dy = normal(g, 9, 3, 64, dtype=torch.float32), normal(g, 9, 3, 64, dtype=torch.float32)
    pos = torch.randint(0, 4000, (9,), device=DEV, generator=g, dtype=torch.int32)
    dx = torch.empty_like(x)
    ctx.rotary(crf.Rope(64, **a), pos, dy, dx, inverse=True)
    leaf = x.double().requires_grad_()
    rotate = lambda t: rotate64(t, pos, 64, a)[0]  # noqa: E731
    want = torch.autograd.grad((rotate(leaf) * dy.double()).sum(), leaf)[0]
    _, size = rotate64(dy, pos, 64, a)
    assert bool(((dx.double() - want).abs() <= 2.0**-24 * want.abs() + 2.0**-21 * size).all())
    # and differences of the call itself along one direction: the map is linear
    e = normal(g, 9, 3, 64, dtype=torch.float32)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    ctx.rotary(crf.Rope(64, **a), pos, x - e, y0)
    ctx.rotary(crf.Rope(64, **a), pos, x + e, y1)
    lhs = ((y1.double() - y0.double()) / 2 * dy.double()).sum()
    rhs = (dx.double() * e.double()).sum()
    # 1728 terms of size about 1.2^2, each off by a few 2^-22
    assert abs(float(lhs - rhs)) <= 1728 * 8 * 2.0**-22


# ---------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("name,layout", [("whole", "half"), ("bands", "half"), ("part", "interleaved"), (None, None)])
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (28, 4, 128), (3, 3, 64)])
def test_append_writes_its_slots_only(ctx, hq, hkv, dim, name, layout):
    g = gen(6)
    new, pos = [1, 40, 0, 17, 1], [0, 31, 5, 16, 777]
    tables, total = tables_of(g, [pages_for(m + p) for m, p in zip(new, pos)])
    kp, vp = normal(g, total, hkv, PAGE, dim), normal(g, total, hkv, PAGE, dim)
    kp0, vp0 = kp.clone(), vp.clone()
    rows = sum(new)
    qkv = normal(g, rows, hq + 2 * hkv, dim)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    at = torch.cat([torch.arange(p, p + m) for m, p in zip(new, pos)]).to(DEV)
    req = torch.cat([torch.full((m,), i) for i, m in enumerate(new)])
    page = torch.stack([tables[i][p // PAGE] for i, p in zip(req.tolist(), at.tolist())]).long()
    chunks = crf.Chunks(tables, new, pos)
    a = None if name is None else dict(ROPES[name], layout=layout)
    q_out = torch.empty(rows, hq, dim, dtype=BF16, device=DEV)
    pool = crf.KVPool([torch.zeros_like(kp), kp], [torch.zeros_like(vp), vp])
    if a is None:
        ctx.cache_append(pool, 1, chunks, k, v)
        assert torch.equal(kp[page, :, at % PAGE], k)
    else:
        ctx.cache_append(pool, 1, chunks, k, v, q=q, q_out=q_out, rope=crf.Rope(dim, **a))
        assert_rotated(kp[page, :, at % PAGE], k, at, dim, a)
        assert_rotated(q_out, q, at, dim, a)
    ctx.check()
    assert torch.equal(vp[page, :, at % PAGE], v)
    kp[page, :, at % PAGE] = kp0[page, :, at % PAGE]
    vp[page, :, at % PAGE] = vp0[page, :, at % PAGE]
    assert torch.equal(kp, kp0) and torch.equal(vp, vp0)
    assert not pool.k_pages[0].any() and not pool.v_pages[0].any()


def test_append_leaves_out_pages_outside_the_pool(ctx):
    g = gen(7)
    kp, vp = normal(g, 4, 2, PAGE, 64), normal(g, 4, 2, PAGE, 64)
    kp0, vp0 = kp.clone(), vp.clone()
    k, v = normal(g, 20, 2, 64), normal(g, 20, 2, 64)
    pool = crf.KVPool([kp], [vp])
    for bad in (4, -1, 2**31 - 1, -(2**31)):
        ctx.cache_append(pool, 0, crf.Chunks([ints(2, bad)], [20], [0]), k, v)
        with pytest.raises(CrfError, match="EINVAL"):
            ctx.check()
        assert torch.equal(kp[2].transpose(0, 1), k[:16]) and torch.equal(vp[2].transpose(0, 1), v[:16])
        kp[2], vp[2] = kp0[2], vp0[2]
        assert torch.equal(kp, kp0) and torch.equal(vp, vp0)
    ctx.check()


# ---------------------------------------------------------------------------------------------- attention
class Setup:
    """Seeded pages, tables and rows; every slot that no row sees holds NaN or an infinity."""

    def __init__(self, seed, hq, hkv, dim, chunks, causal=True, window=0, poison=True, scale_q=1.0):
        g = gen(seed)
        self.hq, self.hkv, self.dim, self.causal, self.window = hq, hkv, dim, causal, window
        self.chunks = [c if len(c) == 3 else (*c, c[0] + c[1]) for c in chunks]  # (rows, position, keys)
        self.tables, total = tables_of(g, [pages_for(c[2]) for c in self.chunks])
        shape = (total, hkv, PAGE, dim)
        k, v = normal(g, *shape), (normal(g, *shape, dtype=torch.float32) + 0.5).to(BF16)
        if poison:
            self.k = torch.full(shape, math.nan, dtype=BF16, device=DEV)
            self.v = torch.full(shape, math.nan, dtype=BF16, device=DEV)
            self.k[:, :, ::2], self.v[:, :, ::2] = math.inf, -math.inf
            for (m, p, n), t in zip(self.chunks, self.tables):
                seen = self.visible(m, p, n).any(0).nonzero().squeeze(1)
                page = t.long()[seen // PAGE]
                self.k[page, :, seen % PAGE] = k[page, :, seen % PAGE]
                self.v[page, :, seen % PAGE] = v[page, :, seen % PAGE]
        else:
            self.k, self.v = k, v
        self.rows = sum(c[0] for c in self.chunks)
        self.q = (normal(g, self.rows, hq, dim, dtype=torch.float32) * scale_q).to(BF16)
        self.pool = crf.KVPool([self.k], [self.v])

    def visible(self, m, p, n):
        j, at = torch.arange(n, device=DEV), torch.arange(p, p + m, device=DEV)[:, None]
        seen = torch.ones(m, n, dtype=torch.bool, device=DEV)
        if self.causal:
            seen &= j <= at
        if self.window:
            seen &= j > at - self.window
        return seen

    def batch(self):
        return crf.Chunks(self.tables, [c[0] for c in self.chunks], [c[1] for c in self.chunks], [c[2] for c in self.chunks])

    def run(self, ctx, scale=0.0, q=None, out=None, stream=None):
        b = self.batch()
        q = self.q if q is None else q
        out = torch.full((self.rows, self.hq, self.dim), 7.0, dtype=BF16, device=DEV) if out is None else out
        lse = torch.full((self.rows, self.hq), 7.0, device=DEV)
        ws = ctx.chunk_attention_workspace(self.pool, b, self.hq, causal=self.causal, window=self.window)
        ctx.chunk_attention(self.pool, 0, b, q, out, ws, lse=lse, scale=scale, causal=self.causal, window=self.window, stream=stream)
        return out, lse

    def verify(self, out, lse, scale=0.0):
        scale = scale or self.dim**-0.5
        row = 0
        for (m, p, n), t in zip(self.chunks, self.tables):
            if m == 0:
                continue
            seen = self.visible(m, p, n)
            k = self.k[t.long()].transpose(1, 2).reshape(-1, self.hkv, self.dim)[:n].double()
            v = self.v[t.long()].transpose(1, 2).reshape(-1, self.hkv, self.dim)[:n].double()
            some = seen.any(0)
            k, v = torch.where(some[:, None, None], k, 0.0), torch.where(some[:, None, None], v, 0.0)
            grp = self.hq // self.hkv
            for h in range(self.hq):
                q = self.q[row:row + m, h].double()
                kk, vv = k[:, h // grp], v[:, h // grp]
                z = (q @ kk.T * scale).masked_fill(~seen, -math.inf)
                top = z.amax(1, keepdim=True) if n else torch.full((m, 1), -math.inf, device=DEV, dtype=torch.float64)
                e = (z - torch.where(top.isinf(), 0.0, top)).exp()
                l = e.sum(1, keepdim=True)
                w = e / torch.where(l > 0, l, 1.0)
                want, size = w @ vv, w @ vv.abs()
                got = out[row:row + m, h].double()
                tol = size * (2.0**-8 + 2.0**-12) + want.abs() * 2.0**-8 * 1.01
                assert bool(((got - want).abs() <= tol).all()), (h, float(((got - want).abs() - tol).max()))
                lse64 = (top + l.log()).squeeze(1)
                gl = lse[row:row + m, h].double()
                empty = ~seen.any(1)
                assert bool((gl[empty] == -math.inf).all()) and bool((got[empty] == 0).all())
                reach = (q.abs() @ kk.abs().T * scale).masked_fill(~seen, 0.0).amax(1) if n else torch.zeros(m, device=DEV)
                assert bool(((gl - lse64).abs() <= 2.0**-16 * reach + 2.0**-17 * (1 + lse64.abs()))[~empty].all()), h
            row += m


HEADS = [(4, 2, 64), (12, 2, 128), (28, 4, 128), (5, 5, 64), (16, 1, 128), (40, 2, 64)]
# (rows, position[, keys])
BATCHES = {
    "one token, no cache": [(1, 0)], "one token": [(1, 299)], "one token, page ends": [(1, 15), (1, 16), (1, 127), (1, 128), (1, 129)],
    "one token, long": [(1, 5000), (1, 3)], "drafts": [(5, 200), (8, 0), (3, 1021)], "chunk from nothing": [(130, 0)],
    "chunk": [(100, 333)], "odd": [(257, 129), (1, 700), (17, 15)], "empty requests": [(0, 50), (3, 40), (0, 0), (2, 9)],
    "no keys": [(4, 10, 0), (2, 20, 0)], "fewer keys than positions": [(20, 100, 90), (4, 2, 1)], "keys behind the rows": [(6, 10, 300)],
}


@pytest.mark.parametrize("batch", sorted(BATCHES))
@pytest.mark.parametrize("hq,hkv,dim", HEADS)
def test_attention_batches(ctx, hq, hkv, dim, batch):
    s = Setup(11, hq, hkv, dim, BATCHES[batch])
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("window", [1, 16, 100, 128, 129, 1000])
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (28, 4, 128), (5, 5, 64)])
def test_attention_windows(ctx, hq, hkv, dim, window):
    # the last request's rows have left their window of the cached keys behind, in part or whole
    s = Setup(12, hq, hkv, dim, [(1, 2000), (70, 300), (300, 130), (5, 0), (12, 400, max(0, 410 - window)), (3, 700, 100)], window=window)
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (12, 2, 128)])
def test_attention_without_causality(ctx, hq, hkv, dim):
    s = Setup(13, hq, hkv, dim, [(1, 0, 200), (90, 10, 400), (3, 7, 1), (2, 5, 0)], causal=False)
    s.verify(*s.run(ctx))
    s = Setup(14, hq, hkv, dim, [(9, 300, 500), (4, 600, 90)], causal=False, window=64)
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("scale_q", [0.0, 8.0, 60.0])
def test_attention_of_sharp_and_flat_scores(ctx, scale_q):
    s = Setup(15, 12, 2, 128, [(40, 500), (1, 3000)], scale_q=scale_q)
    s.verify(*s.run(ctx))
    s.verify(*s.run(ctx, scale=0.01), scale=float(np.float32(0.01)))


def test_attention_rising_scores(ctx):
    """Keys whose scores rise along the cache: the running maximum grows in every tile."""
    s = Setup(16, 4, 2, 64, [(150, 900), (1, 1500)], poison=False)
    for (m, p, n), t in zip(s.chunks, s.tables):
        up = torch.arange(n, device=DEV) / 40.0
        page, slot = t.long()[torch.arange(n, device=DEV) // PAGE], torch.arange(n, device=DEV) % PAGE
        s.k[page, :, slot] = (s.k[page, :, slot].float() * 0.1 + up[:, None, None]).to(BF16)
    s.q.copy_((s.q.float().abs() * 0.5).to(BF16))
    s.verify(*s.run(ctx))


def test_attention_many_requests(ctx):
    g = np.random.default_rng(3)
    c = [(int(g.integers(0, 20)), int(g.integers(0, 400))) for _ in range(crf.abi.MAX_CHUNKS)]
    s = Setup(17, 4, 2, 64, c)
    s.verify(*s.run(ctx))
    ctx.check()


def test_attention_long_chunk(ctx):
    s = Setup(18, 12, 2, 128, [(700, 2100), (513, 0), (1, 9000)])
    s.verify(*s.run(ctx))
    s = Setup(19, 4, 4, 64, [(1100, 77)])
    s.verify(*s.run(ctx))
    ctx.check()


@pytest.mark.parametrize("hq,hkv,dim,chunks", [
    (28, 4, 128, [(16, 20000)]), (12, 2, 128, [(9, 30001), (1, 100)]), (4, 2, 64, [(60, 25000)]), (5, 5, 64, [(100, 9000), (128, 7000)]),
    (28, 4, 128, [(300, 12000), (2, 9000), (18, 11111)]), (4, 2, 64, [(700, 3000)]), (16, 1, 128, [(8, 40000), (40, 5000)]),
])
def test_attention_cut_items(ctx, hq, hkv, dim, chunks):
    """Few query tiles over many keys: every item is cut among CTAs, whatever the number of rows in its tile."""
    s = Setup(25, hq, hkv, dim, chunks)
    out, lse = s.run(ctx)
    s.verify(out, lse)
    for _ in range(3):
        again, lse2 = s.run(ctx)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    ctx.check()


def test_attention_values_that_only_later_rows_see(ctx):
    """NaN and infinities in keys' values reach the rows that see them and no other."""
    for hq, hkv, dim in ((4, 2, 64), (28, 4, 128)):
        for m, p, at in ((40, 300, 320), (200, 100, 250), (6, 10, 12)):
            s = Setup(20, hq, hkv, dim, [(m, p)], poison=False)
            page, slot = s.tables[0].long()[at // PAGE], at % PAGE
            s.v[page, 0, slot, 3], s.v[page, 0, slot, 5] = math.nan, math.inf
            out, lse = s.run(ctx)
            grp, first = hq // hkv, at - p
            assert bool(out[first:, :grp, 3].isnan().all()) and bool((out[first:, :grp, 5] == math.inf).all())
            clean = out.clone()
            clean[first:, :grp, 3] = clean[first:, :grp, 5] = 0
            assert bool(clean.isfinite().all())
            s.v[page, 0, slot, 3] = s.v[page, 0, slot, 5] = 0
            out2, lse2 = s.run(ctx)
            out2[first:, :grp, 3] = out2[first:, :grp, 5] = 0
            assert torch.equal(clean, out2) and torch.equal(lse, lse2)
    ctx.check()


def test_attention_strides_and_rows_behind(ctx):
    s = Setup(21, 12, 2, 128, [(33, 90), (1, 400)])
    want, lse0 = s.run(ctx)
    wide = torch.full((40, 16, 136), 9.0, dtype=BF16, device=DEV)
    q = torch.zeros(36, 14, 136, dtype=BF16, device=DEV)[1:35, 1:13, :128]
    q.copy_(s.q)
    out = wide[2:36, 3:15, 8:]
    got, lse = s.run(ctx, q=q, out=out)
    assert torch.equal(out, want) and torch.equal(lse, lse0)
    out.fill_(9.0)
    assert bool((wide == 9.0).all())
    # heads outside, rows inside
    q = s.q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty(12, 34, 128, dtype=BF16, device=DEV).transpose(0, 1)
    s.run(ctx, q=q, out=out)
    assert torch.equal(out, want)


def test_strides_of_axes_of_one_are_not_read(ctx):
    # one row, or one head: a tensor may carry any stride there
    def odd(t, row, head):
        return t.as_strided(t.shape, (row, head, 1))

    s = Setup(23, 8, 2, 128, [(1, 300)])
    want, _ = s.run(ctx)
    out = torch.empty_like(s.q)
    got, _ = s.run(ctx, q=odd(s.q, 3, 128), out=odd(out, 5, 128))
    assert torch.equal(got, want)
    s = Setup(24, 1, 1, 64, [(37, 300)])
    want, _ = s.run(ctx)
    out = torch.empty_like(s.q)
    got, _ = s.run(ctx, q=odd(s.q, 64, 1), out=odd(out, 64, 0))
    assert torch.equal(got, want)
    x, pos = normal(gen(25), 1, 8, 64), ints(77)
    want, got = torch.empty_like(x), torch.empty_like(x)
    ctx.rotary(crf.Rope(64), pos, x, want)
    ctx.rotary(crf.Rope(64), pos, odd(x, 0, 64), odd(got, 1, 64))
    assert torch.equal(got, want)
    pool = [torch.zeros(2, 1, 16, 64, dtype=BF16, device=DEV) for _ in range(4)]
    k, q = normal(gen(26), 1, 1, 64), normal(gen(27), 1, 1, 64)
    q_out = torch.empty_like(q)
    c = crf.Chunks([ints(1)], [1], [3])
    rope = crf.Rope(64)
    ctx.cache_append(crf.KVPool(pool[:1], pool[1:2]), 0, c, k, k, q=q.clone(), rope=rope)
    ctx.cache_append(crf.KVPool(pool[2:3], pool[3:]), 0, c, odd(k, 1, 7), odd(k, 0, 0), q=odd(q, 1, 1), q_out=odd(q_out, 0, 0),
                     rope=rope)
    ctx.rotary(rope, ints(3), q)
    assert torch.equal(pool[0], pool[2]) and torch.equal(pool[1], pool[3]) and torch.equal(q_out, q)
    ctx.check()


def test_attention_shared_pages_and_same_bits(ctx):
    s = Setup(22, 28, 4, 128, [(1, 2000), (1, 1500), (9, 700)])
    s.tables = [s.tables[0]] * 3  # three requests on one prefix
    a, la = s.run(ctx)
    b, lb = s.run(ctx)
    assert torch.equal(a, b) and torch.equal(la, lb)
    s.k, s.v = torch.nan_to_num(s.k, 0, 0, 0), torch.nan_to_num(s.v, 0, 0, 0)
    s.pool = crf.KVPool([s.k], [s.v])
    s.verify(*s.run(ctx))


def test_attention_bad_pages_are_reported(ctx):
    s = Setup(23, 4, 2, 64, [(3, 40), (2, 30)], poison=False)
    good, _ = s.run(ctx)
    for bad in (-1, s.k.shape[0], 2**31 - 1, -(2**31)):
        s.tables = [s.tables[0].clone(), s.tables[1]]
        keep = int(s.tables[0][1])
        s.tables[0][1] = bad
        out, _ = s.run(ctx)
        with pytest.raises(CrfError, match="EINVAL"):
            ctx.check()
        assert torch.equal(out[3:], good[3:])  # the other request
        s.tables[0][1] = keep
    out, _ = s.run(ctx)
    ctx.check()
    assert torch.equal(out, good)


# ---------------------------------------------------------------------------------------------- pages
class Pool:
    def __init__(self, seed, tokens, free, layers=3, hkv=2, dim=64, share=True):
        g = gen(seed)
        counts = [pages_for(n) for n in tokens]
        self.tables, self.total = tables_of(g, counts, free)
        if share:
            for i in range(1, len(tokens), 2):
                n = min(counts[i], counts[i - 1]) // 2
                self.tables[i][:n] = self.tables[i - 1][:n]
        self.tokens, self.layers = tokens, layers
        self.refs = torch.zeros(self.total, dtype=torch.int32, device=DEV)
        for t in self.tables:
            self.refs.index_add_(0, t.long(), torch.ones_like(t))
        self.k = normal(g, layers, self.total, hkv, PAGE, dim)
        self.v = normal(g, layers, self.total, hkv, PAGE, dim)
        self.pool = crf.KVPool(list(self.k), list(self.v))

    def page_tables(self, outs=None):
        outs = [torch.full_like(t, -7) for t in self.tables] if outs is None else outs
        return crf.PageTables(self.tables, self.tokens, outs), outs


def fork_model(tables, tokens, refs, k, v, deep):
    refs, free = list(refs), [p for p, r in enumerate(refs) if r == 0]
    k, v, out = k.clone(), v.clone(), []
    for t, n in zip(tables, tokens):
        child = []
        for i in range(pages_for(n)):
            live = min(PAGE, n - PAGE * i)
            if deep or live < PAGE:
                p = free.pop(0)
                k[:, p, :, :live], v[:, p, :, :live] = k[:, t[i], :, :live], v[:, t[i], :, :live]
                refs[p] = 1
            else:
                p = t[i]
                refs[p] += 1
            child.append(p)
        out.append(child)
    return out, refs, k, v


@pytest.mark.parametrize("deep", [False, True])
@pytest.mark.parametrize("tokens,free", [([40], 4), ([16], 1), ([1], 1), ([0, 33, 0], 9), ([500, 300, 16, 15, 17], 70),
                                         ([5] * 90, 95)])
def test_pages_fork(ctx, tokens, free, deep):
    s = Pool(31, tokens, free)
    lists = [t.tolist() for t in s.tables]
    want, refs, k, v = fork_model(lists, tokens, s.refs.tolist(), s.k, s.v, deep)
    tables, outs = s.page_tables()
    refs_out = torch.full_like(s.refs, -9)
    before = s.refs.clone()
    ws = ctx.pages_workspace(s.total, tables)
    ctx.pages_fork(s.pool, s.refs, tables, ws, refs_out=refs_out, deep=deep)
    ctx.check()
    assert [o.tolist() for o in outs] == want and refs_out.tolist() == refs and torch.equal(s.refs, before)
    assert torch.equal(s.k, k) and torch.equal(s.v, v)
    assert [t.tolist() for t in s.tables] == lists
    # in place, a second generation
    want2, refs2, k2, v2 = fork_model(lists, tokens, refs, k, v, False) if sum(r == 0 for r in refs) >= sum(n % 16 > 0 for n in tokens) \
        else (None,) * 4
    if want2 is not None:
        ctx.pages_fork(s.pool, refs_out, tables, ws)
        ctx.check()
        assert [o.tolist() for o in outs] == want2 and refs_out.tolist() == refs2 and torch.equal(s.k, k2) and torch.equal(s.v, v2)


def assert_rejected(ctx, s, call, match, outs=(), extra=()):
    """The call is reported, and nothing outside its workspace was written."""
    tensors = [s.k, s.v, s.refs, *s.tables, *outs, *extra]
    before = [t.clone() for t in tensors]
    call()
    with pytest.raises(CrfError, match=match):
        ctx.check()
    ctx.check()
    assert all(torch.equal(a, b) for a, b in zip(tensors, before))


def test_pages_fork_rejects(ctx):
    s = Pool(32, [100, 40], 1)
    tables, outs = s.page_tables()
    ws = ctx.pages_workspace(s.total, tables)
    refs_out = torch.full_like(s.refs, -9)
    fork = lambda **kw: (lambda: ctx.pages_fork(s.pool, s.refs, tables, ws, **kw))  # noqa: E731
    free = int((s.refs == 0).sum())
    assert free < 7 + 3
    assert_rejected(ctx, s, fork(refs_out=refs_out, deep=True), "ENOMEM", outs, [refs_out])
    for bad in (-1, s.total, 2**31 - 1):
        keep = int(s.tables[1][2])
        s.tables[1][2] = bad
        assert_rejected(ctx, s, fork(refs_out=refs_out), "EINVAL", outs, [refs_out])
        s.tables[1][2] = keep
    keep = s.refs.clone()
    s.refs[int(s.tables[0][3])] = 0  # a page that nothing holds
    assert_rejected(ctx, s, fork(), "EINVAL", outs)
    s.refs.copy_(keep)
    s.refs[(keep == 0).nonzero()[0]] = -1
    assert_rejected(ctx, s, fork(), "EINVAL", outs)
    s.refs.copy_(keep)


def compact_model(tables, refs, k, v):
    live = [p for p, r in enumerate(refs) if r > 0]
    n = len(live)
    holes, movers = [p for p in range(n) if refs[p] == 0], [p for p in live if p >= n]
    to = dict(zip(movers, holes))
    k, v, out = k.clone(), v.clone(), [0] * len(refs)
    for p in live:
        out[to.get(p, p)] = refs[p]
    k[:, holes], v[:, holes] = k[:, movers], v[:, movers]
    return [[to.get(p, p) for p in t] for t in tables], out, k, v


@pytest.mark.parametrize("tokens,free", [([40], 4), ([16], 1), ([16], 0), ([0, 33, 0], 9), ([500, 300, 16, 15, 17], 70),
                                         ([5] * 90, 200), ([2000, 3000, 1000, 900], 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_pages_compact(ctx, tokens, free, in_place):
    s = Pool(33, tokens, free, layers=2)
    lists = [t.tolist() for t in s.tables]
    want, refs, k, v = compact_model(lists, s.refs.tolist(), s.k, s.v)
    tables, outs = s.page_tables(s.tables if in_place else None)
    refs_out = None if in_place else torch.full_like(s.refs, -9)
    ws = ctx.pages_workspace(s.total, tables)
    ctx.pages_compact(s.pool, s.refs, tables, ws, refs_out=refs_out)
    ctx.check()
    assert [o.tolist() for o in outs] == want and (s.refs if in_place else refs_out).tolist() == refs
    assert torch.equal(s.k, k) and torch.equal(s.v, v)


def test_pages_compact_rejects(ctx):
    s = Pool(34, [100, 40, 70], 30)
    tables, outs = s.page_tables()
    ws = ctx.pages_workspace(s.total, tables)
    refs_out = torch.full_like(s.refs, -9)
    compact = lambda: ctx.pages_compact(s.pool, s.refs, tables, ws, refs_out=refs_out)  # noqa: E731
    # a reference that no table of the call holds
    missing = crf.PageTables(s.tables[:2], s.tokens[:2], outs[:2])
    assert_rejected(ctx, s, lambda: ctx.pages_compact(s.pool, s.refs, missing, ws, refs_out=refs_out), "EINVAL", outs, [refs_out])
    keep = s.refs.clone()
    s.refs[int(s.tables[0][3])] += 1
    assert_rejected(ctx, s, compact, "EINVAL", outs, [refs_out])
    s.refs.copy_(keep)
    for bad in (-1, s.total, -(2**31)):
        last = int(s.tables[2][4])
        s.tables[2][4] = bad
        assert_rejected(ctx, s, compact, "EINVAL", outs, [refs_out])
        s.tables[2][4] = last
    compact()
    ctx.check()


@pytest.mark.parametrize("tokens,free", [([40], 4), ([1], 0), ([0, 33, 0], 9), ([500, 300, 16, 15, 17], 70), ([5] * 500, 3)])
def test_pages_release(ctx, tokens, free):
    s = Pool(35, tokens, free, layers=1)
    want = s.refs.clone()
    s.refs += 1
    tables = crf.PageTables(s.tables, s.tokens)
    ws = ctx.pages_workspace(s.total, tables)
    out = torch.full_like(s.refs, -9)
    ctx.pages_release(s.refs, tables, ws, refs_out=out)
    assert torch.equal(out, torch.ones_like(out)) and torch.equal(s.refs, want + 1)
    twice = crf.PageTables(s.tables[:1] * 2, [tokens[0]] * 2)  # the same table twice
    n = len(s.tables[0])
    s.refs[s.tables[0].long()] = 5
    before = s.refs.clone()
    ctx.pages_release(s.refs, twice, ctx.pages_workspace(s.total, twice))
    ctx.check()
    before[s.tables[0].long()] = 3
    assert torch.equal(s.refs, before) and n == pages_for(tokens[0])


def test_pages_release_rejects(ctx):
    s = Pool(36, [100, 40, 70], 30)
    twice = crf.PageTables([s.tables[0], s.tables[2], s.tables[2]], [100, 70, 70])
    ws = ctx.pages_workspace(s.total, twice)
    assert_rejected(ctx, s, lambda: ctx.pages_release(s.refs, twice, ws), "EINVAL")
    tables, _ = s.page_tables()
    for bad in (-1, s.total, 2**31 - 1):
        last = int(s.tables[2][4])
        s.tables[2][4] = bad
        assert_rejected(ctx, s, lambda: ctx.pages_release(s.refs, tables, ws), "EINVAL")
        s.tables[2][4] = last
    ctx.pages_release(s.refs, tables, ws)
    ctx.check()
    assert not s.refs.any()


# ---------------------------------------------------------------------------------------------- together
def test_calls_on_other_streams_and_captured(ctx):
    """Every call on a stream of its own and captured into a graph, replayed on new contents."""
    s = Setup(41, 12, 2, 128, [(5, 700), (1, 3000)], poison=False)
    p = Pool(42, [100, 40], 20)
    tables, outs = p.page_tables()
    pws, refs_out = ctx.pages_workspace(p.total, tables), torch.empty_like(p.refs)
    b = s.batch()
    ws = ctx.chunk_attention_workspace(s.pool, b, s.hq)
    rope = crf.Rope(128, theta=1e6)
    x, k, v = (normal(gen(43 + i), s.rows, h, 128) for i, h in enumerate((12, 2, 2)))
    q, out, lse = torch.empty_like(x), torch.empty_like(x), torch.empty(s.rows, 12, device=DEV)
    pos = torch.cat([torch.arange(c[1], c[1] + c[0], dtype=torch.int32) for c in s.chunks]).to(DEV)
    y = torch.empty_like(x)

    def calls():
        ctx.cache_append(s.pool, 0, b, k, v, q=x, q_out=q, rope=rope)
        ctx.chunk_attention(s.pool, 0, b, q, out, ws, lse=lse)
        ctx.rotary(rope, pos, x, y)
        ctx.pages_fork(p.pool, p.refs, tables, pws, refs_out=refs_out, deep=True)

    keep = [t.clone() for t in (s.k, s.v, p.k, p.v)]
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (q, out, lse, y, s.k, s.v, refs_out, p.k, p.v, *outs)]
    got = lambda: (q, out, lse, y, s.k, s.v, refs_out, p.k, p.v, *outs)  # noqa: E731

    def reset():
        for t, o in zip((s.k, s.v, p.k, p.v), keep):
            t.copy_(o)
        for t in (q, out, lse, y, refs_out, *outs):
            t.fill_(3)

    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(2):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got(), want))
    # new contents, same addresses
    x.mul_(0.5)
    reset()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, (want[3].float() * 0.5).to(BF16)) and not torch.equal(out, want[1])
    ctx.check()


@pytest.mark.parametrize("captured", [False, True])
def test_calls_see_what_was_just_written(ctx, captured):
    """Inputs made by a copy, a fill and a kernel right before each call, on two joined streams; every kernel of these
    calls may become resident early, and none may read early."""
    s = Setup(44, 12, 2, 128, [(3, 700), (1, 2500)], poison=False)
    p = Pool(45, [100, 40], 20, layers=1)
    tables, outs = p.page_tables()
    pws, refs2 = ctx.pages_workspace(p.total, tables), torch.empty_like(p.refs)
    b = s.batch()
    ws = ctx.chunk_attention_workspace(s.pool, b, s.hq)
    rope = crf.Rope(128, theta=1e6)
    src = [normal(gen(46 + i), s.rows, h, 128) for i, h in enumerate((12, 2, 2))]
    x, k, v = (torch.empty_like(t) for t in src)
    q, out, lse, refs = torch.empty_like(x), torch.empty_like(x), torch.empty(s.rows, 12, device=DEV), torch.empty_like(p.refs)
    counts, side = p.refs.clone(), torch.cuda.Stream()
    big = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)

    def calls():
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            big.fill_(1)                      # a while
            refs.copy_(counts)                # device to device
            ctx.pages_fork(p.pool, refs, tables, pws, refs_out=refs2)
            k.copy_(src[1])
        x.zero_()
        x.add_(src[0])                        # a kernel
        v.copy_(src[2])
        here.wait_stream(side)
        ctx.cache_append(s.pool, 0, b, k, v, q=x, q_out=q, rope=rope)
        ctx.chunk_attention(s.pool, 0, b, q, out, ws, lse=lse)
        out.mul_(2)                           # and a kernel behind

    calls()
    torch.cuda.synchronize()
    first = [t.clone() for t in (q, out, lse, refs2, *outs)]
    assert torch.equal(refs2, fork_counts(p, counts))
    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
    for i in range(20):
        for t in (x, k, v, q, out, lse, refs, refs2, *outs):
            t.fill_(i)
        for t in src:
            t.neg_()
        counts[p.tables[0].long()[0]] += 1
        graph.replay() if captured else calls()
        torch.cuda.synchronize()
        # q and k change their signs together: the same scores, the values' signs turned for the new rows alone
        assert torch.equal(q, first[0] if i % 2 else -first[0])
        assert torch.equal(refs2, fork_counts(p, counts)) and all(torch.equal(a, c) for a, c in zip(outs, first[4:]))
        if i % 2:
            assert torch.equal(out, first[1]) and torch.equal(lse, first[2])
    ctx.check()


def fork_counts(p, refs):
    """Counts after a shallow fork of the pool's tables."""
    out, free = refs.clone(), (refs == 0).nonzero().squeeze(1)
    fresh = 0
    for t, n in zip(p.tables, p.tokens):
        out.index_add_(0, t[: n // PAGE].long(), torch.ones_like(t[: n // PAGE]))
        fresh += n % PAGE > 0
    out[free[:fresh]] = 1
    return out


def test_calls_at_the_end_of_a_large_pool(ctx):
    """Pages whose elements lie behind 2^31: a layer's pool of 4.5 GB."""
    hq, hkv, dim, pages = 28, 4, 128, 275000
    assert pages * hkv * PAGE * dim > 2**31
    kp, vp = (torch.empty(pages, hkv, PAGE, dim, dtype=BF16, device=DEV) for _ in range(2))
    g = gen(47)
    table = ints(pages - 1, pages - 7, 3, pages - 2, pages - 3)
    n, m = 70, 9
    k, v = normal(g, n, hkv, dim), normal(g, n, hkv, dim)
    pool = crf.KVPool([kp], [vp])
    ctx.cache_append(pool, 0, crf.Chunks([table], [n], [0]), k, v)
    at = torch.arange(n, device=DEV)
    assert torch.equal(kp[table.long()[at // PAGE], :, at % PAGE], k)
    assert torch.equal(vp[table.long()[at // PAGE], :, at % PAGE], v)
    q, out = normal(g, m, hq, dim), torch.empty(m, hq, dim, dtype=BF16, device=DEV)
    b = crf.Chunks([table], [m], [n - m])
    ctx.chunk_attention(pool, 0, b, q, out, ctx.chunk_attention_workspace(pool, b, hq))
    z = torch.einsum("mgrd,ngd->mgrn", q.double().view(m, hkv, -1, dim), k.double()) * dim**-0.5
    z = z.masked_fill((at > torch.arange(n - m, n, device=DEV)[:, None])[:, None, None], -math.inf)
    w = z.softmax(-1)
    want = torch.einsum("mgrn,ngd->mgrd", w, v.double()).reshape(m, hq, dim)
    size = torch.einsum("mgrn,ngd->mgrd", w, v.double().abs()).reshape(m, hq, dim)
    assert bool(((out.double() - want).abs() <= size * (2.0**-8 + 2.0**-12) + want.abs() * 2.0**-8 * 1.01).all())
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[:-60] = 1  # nearly full: the new pages are the last ones
    refs[table.long()] = 1
    child = torch.empty_like(table)
    t = crf.PageTables([table], [n], [child])
    free = (refs == 0).nonzero().squeeze(1)
    ctx.pages_fork(pool, refs, t, ctx.pages_workspace(pages, t), deep=True)
    ctx.check()
    assert torch.equal(child.long(), free[:5])
    assert torch.equal(kp[child.long()[at // PAGE], :, at % PAGE], k) and torch.equal(vp[child.long()[at // PAGE], :, at % PAGE], v)


def test_one_parent_forked_twice_in_a_call(ctx):
    s = Pool(48, [100, 40], 20, layers=2)
    lists = [s.tables[0].tolist()] * 2
    want, refs, k, v = fork_model(lists, [100, 100], s.refs.tolist(), s.k, s.v, False)
    outs = [torch.full_like(s.tables[0], -7) for _ in range(2)]
    t = crf.PageTables([s.tables[0]] * 2, [100, 100], outs)
    ctx.pages_fork(s.pool, s.refs, t, ctx.pages_workspace(s.total, t))
    ctx.check()
    assert [o.tolist() for o in outs] == want and s.refs.tolist() == refs and torch.equal(s.k, k) and torch.equal(s.v, v)


def test_continuation_matches_recomputation(ctx):
    """A prefix's cache from crf_recompute_window, extended by new rows layer by layer with these calls, against the
    window call over the whole: the same rotation, layout and attention."""
    import synth
    from tests.harness import DeviceAdapter, DeviceModel, make_pool, split_page_tables
    from tests.gpu_util import REL_KVH, rel_frob, request_kv, to_np
    cfg, n, m = synth.TINY, 203, 70
    dm, ad = DeviceModel(cfg, DEV), DeviceAdapter(cfg, synth.LORA_TINY, 1, DEV)
    total = pages_for(n + m) + 4
    tokens = synth.token_ids(cfg, n + m).to(DEV)
    table = split_page_tables([n + m], total, seed=5, device=DEV)[0]
    whole, part = make_pool(cfg, total, DEV, fill="zeros"), make_pool(cfg, total, DEV, fill="zeros")
    H = [torch.empty(n + m, cfg.hidden, dtype=BF16, device=DEV) for _ in range(cfg.n_layers)]
    for pool, count, hidden in ((whole, n + m, H), (part, n, None)):
        r = crf.Request(table, 0, cfg.n_layers, n_tokens=count, tokens=tokens, hidden_out=hidden)
        ctx.recompute_window(dm.crf, ad.crf, pool, [r], ctx.workspace(dm.crf, ad.crf, [r]))
    ctx.check()
    scale = ad.lcfg.alpha / ad.lcfg.rank

    def project(x, l, name):
        w = dm.layers[l][f"W_{name}"].float()
        if name in ad.layers[l]:
            a, b = ad.layers[l][name]
            w = w + scale * b.float() @ a.float()
        return x.float() @ w.T

    def norm(x, gain):
        x = x.float()
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + cfg.rms_eps) * gain.float()).to(BF16)

    b = crf.Chunks([table], [m], [n])
    rope = crf.Rope(cfg.head_dim, theta=cfg.rope_theta)
    ws = ctx.chunk_attention_workspace(part, b, cfg.n_q_heads)
    x = dm.embed[tokens[n:].long()]
    for l in range(cfg.n_layers):
        y = norm(x, dm.layers[l]["ln1"])
        q, k, v = (project(y, l, name).to(BF16).view(m, -1, cfg.head_dim) for name in "qkv")
        out = torch.empty_like(q)
        ctx.cache_append(part, l, b, k, v, q=q, rope=rope)
        ctx.chunk_attention(part, l, b, q, out, ws)
        x = (x.float() + project(out.view(m, -1), l, "o")).to(BF16)
        y = norm(x, dm.layers[l]["ln2"])
        g = project(y, l, "gate")
        x = (x.float() + project((torch.nn.functional.silu(g) * project(y, l, "up")).to(BF16), l, "down")).to(BF16)
        assert rel_frob(to_np(x), to_np(H[l][n:])) <= REL_KVH, l
        for a, c in ((part.k_pages[l], whole.k_pages[l]), (part.v_pages[l], whole.v_pages[l])):
            assert rel_frob(request_kv(a, table, n + m), request_kv(c, table, n + m)) <= REL_KVH, l
    ctx.check()


def test_two_continuations_of_a_recovered_prefix(ctx):
    """Fork, append, attend, release, compact: two continuations of one prefix against plain caches."""
    g = gen(51)
    hq, hkv, dim, n, layers = 12, 2, 128, 203, 2
    rope, a = crf.Rope(dim, theta=1e6), dict(theta=1e6)
    s = Pool(52, [n, 77], 40, layers=layers, hkv=hkv, dim=dim, share=False)
    # the prefix's pages and room for the continuation's
    room, refs = 64, s.refs
    plain = [[(s.k[l][s.tables[0].long()].transpose(1, 2).reshape(-1, hkv, dim)[:n].clone(),
               s.v[l][s.tables[0].long()].transpose(1, 2).reshape(-1, hkv, dim)[:n].clone()) for l in range(layers)] for _ in range(2)]
    child = torch.empty(pages_for(n + room), dtype=torch.int32, device=DEV)
    parent = torch.empty_like(child)
    parent[:pages_for(n)] = s.tables[0]
    ft = crf.PageTables([parent], [n], [child])
    ctx.pages_fork(s.pool, refs, ft, ctx.pages_workspace(s.total, ft))
    free = (refs == 0).nonzero().squeeze(1).to(torch.int32)
    extra = pages_for(n + room) - pages_for(n)
    parent[pages_for(n):], child[pages_for(n):] = free[:extra], free[extra:2 * extra]
    refs[free[:2 * extra].long()] = 1
    cached = [n, n]
    for new in ([17, 5], [1, 1], [30, 2]):
        rows = sum(new)
        b = crf.Chunks([parent, child], new, cached)
        ws = ctx.chunk_attention_workspace(s.pool, b, hq)
        for l in range(layers):
            x, k, v = normal(g, rows, hq, dim), normal(g, rows, hkv, dim), normal(g, rows, hkv, dim)
            q, out = torch.empty_like(x), torch.empty_like(x)
            ctx.cache_append(s.pool, l, b, k, v, q=x, q_out=q, rope=rope)
            ctx.chunk_attention(s.pool, l, b, q, out, ws)
            row = 0
            for i in range(2):
                m, sl = new[i], slice(row, row + new[i])
                at = torch.arange(cached[i], cached[i] + m, device=DEV)
                kr = rotate64(k[sl], at, dim, a)[0].to(BF16)
                pk, pv = plain[i][l]
                pk, pv = torch.cat([pk, kr]), torch.cat([pv, v[sl]])
                plain[i][l] = (pk, pv)
                z = torch.einsum("mgrd,ngd->mgrn", q[sl].double().view(m, hkv, -1, dim), pk.double()) * dim**-0.5
                z = z.masked_fill((torch.arange(len(pk), device=DEV) > at[:, None])[:, None, None], -math.inf)
                w = z.softmax(-1)
                want = torch.einsum("mgrn,ngd->mgrd", w, pv.double()).reshape(m, hq, dim)
                size = torch.einsum("mgrn,ngd->mgrd", w, pv.double().abs()).reshape(m, hq, dim)
                # as above; and a key's last bit may round the other way here (2^-8 of q k: weights off by a few 2^-8)
                tol = size * 2.0**-6 + want.abs() * 2.0**-8
                assert bool(((out[sl].double() - want).abs() <= tol).all())
                row += m
        cached = [c + m for c, m in zip(cached, new)]
    ctx.check()
    # the parent ends; what is left is packed, and the child's cache reads the same
    rt = crf.PageTables([parent, s.tables[1]], [n + room, 77])
    ctx.pages_release(refs, rt, ctx.pages_workspace(s.total, rt))
    ct = crf.PageTables([child], [n + room], [child])
    ctx.pages_compact(s.pool, refs, ct, ctx.pages_workspace(s.total, ct))
    ctx.check()
    live = pages_for(n + room)
    assert sorted(child.tolist()) == list(range(live)) and refs.tolist() == [1] * live + [0] * (s.total - live)
    for l in range(layers):
        pk, pv = plain[1][l]
        gk = s.k[l][child.long()].transpose(1, 2).reshape(-1, hkv, dim)[:cached[1]]
        gv = s.v[l][child.long()].transpose(1, 2).reshape(-1, hkv, dim)[:cached[1]]
        assert torch.equal(gk[:n], pk[:n]) and torch.equal(gv, pv)
        assert bool(((gk[n:].double() - pk[n:].double()).abs() <= 2.0**-7 * pk[n:].double().abs() + 1e-6).all())
