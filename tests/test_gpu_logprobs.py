"""Log probabilities, entropy, top alternatives and their gradient, against 64-bit formulas.

Tolerances count roundings. With x = (z - max) and W = sum p |x|: a weight 2^(x log2 e) is off by 2^-22 of itself and by
|x| 2^-22 (two roundings of its exponent); under 256 are added in a row, by a lane, a warp, a block and a cluster: 2^-16.
So lse is off by 2^-16 (1 + W) + 2^-22 |lse|, a log probability by 2^-23 |z| more, the entropy (a difference of log s and the
weighted mean of x, which carries the weights' roundings twice) by 2^-15 (1 + W). Gradient: half a step of the type, and
p (|g| + |h| (|l| + |H|)) times 2^-21 + 2^-22 (|l| + |lse|) for p = exp(l), l = z - lse; one 2^-23 |g| at the target; a p under
2^-126, the smallest normal number, is taken as 0, so what multiplies it is off by up to 2^-126 of it. Ids are exact."""
import math

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300.abi import CrfError
from tests.test_gpu_extend import DEV, gen, ints, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


def score(ctx, z, targets=None, k=0, stream=None):
    n = len(z)
    out = dict(lse=torch.full((n,), 7.0, device=DEV), entropy=torch.full((n,), 7.0, device=DEV))
    if targets is not None:
        out["logprob"] = torch.full((n,), 7.0, device=DEV)
    if k:
        out.update(top_ids=torch.full((n, k), -7, dtype=torch.int32, device=DEV), top_logprobs=torch.full((n, k), 7.0, device=DEV))
    ctx.logprobs(z, targets, stream=stream, **out)
    return out


def assert_scored(out, z, targets=None):
    w = z.double()
    n = len(w)
    top = w.amax(1, keepdim=True)
    base = torch.where(top.isinf(), 0.0, top)
    e = (w - base).exp()
    s = e.sum(1)
    empty = s == 0
    lse = (base[:, 0] + s.log())
    p = e / torch.where(empty, 1.0, s)[:, None]
    x = torch.where(p > 0, w - base, 0.0)
    mean = (p * x.abs()).sum(1)
    tol = torch.where(empty, 0.0, 2.0**-16 * (1 + mean) + 2.0**-22 * lse.abs())

    def near(got, want, tol):
        same = (got.double() == want) | (want.isinf() & (got == want))
        assert bool((same | ((got.double() - want).abs() <= tol)).all()), float(((got.double() - want).abs() - tol).nan_to_num().max())

    near(out["lse"], lse, tol)
    near(out["entropy"], torch.where(empty, 0.0, s.clamp(min=1e-300).log() - (p * x).sum(1)), 2.0**-15 * (1 + mean))
    if targets is not None:
        t = targets.long()
        zt = w.gather(1, t.clamp(min=0)[:, None])[:, 0]
        want = torch.where(t < 0, 0.0, torch.where(empty, -math.inf, zt - torch.where(empty, 0.0, lse)))
        near(out["logprob"], want, tol + 2.0**-23 * zt.abs().nan_to_num(posinf=0))
    if "top_ids" in out:
        k = out["top_ids"].shape[1]
        ids = torch.sort(w, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(out["top_ids"].long(), ids)
        z_top = w.gather(1, ids)
        want = torch.where(empty[:, None], -math.inf, z_top - torch.where(empty, 0.0, lse)[:, None])
        near(out["top_logprobs"], want, (tol[:, None] + 2.0**-23 * z_top.abs().nan_to_num(posinf=0, neginf=0)))
    assert n == len(out["lse"])


def logits(g, n, v, dtype, wide=3.0):
    return (normal(g, n, v, dtype=torch.float32) * wide).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 5, 31, 33, 255, 256, 257, 512, 1000, 1024, 1031, 4099, 50001, 151936, 152064])
def test_vocabularies(ctx, vocab, dtype):
    g = gen(1)
    for rows in (1, 3, 20):
        z = logits(g, rows, vocab, dtype)
        t = torch.randint(-1, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
        for k in sorted({0, min(vocab, 1), min(vocab, 20), min(vocab, 32)}):
            assert_scored(score(ctx, z, t, k), z, t)
    ctx.check()


@pytest.mark.parametrize("rows,vocab", [(400, 5003), (700, 50001), (5000, 512), (160, 152064), (80, 20011)])
def test_many_rows(ctx, rows, vocab):
    g = gen(2)
    z = logits(g, rows, vocab, torch.bfloat16)
    t = torch.randint(-1, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    assert_scored(score(ctx, z, t, 8), z, t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("vocab", [1009, 2049, 4097, 8170, 8177])
def test_many_short_rows(ctx, vocab, dtype):
    g = gen(14)
    big = logits(g, 2600, vocab + 5, dtype)
    for first in (0, 3):
        z = big[:, first:first + vocab]
        t = torch.randint(-1, vocab, (2600,), device=DEV, generator=g, dtype=torch.int32)
        for k in (0, 8, 32):
            assert_scored(score(ctx, z, t, k), z, t)
    ctx.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_short_rows_of_ties_and_extremes(ctx, dtype):
    for vocab in (200, 700, 5000):
        z = torch.cat([make_row(name, vocab, dtype) for name in ROWS]).repeat(210, 1)
        for k in (1, 17, 32):
            assert_scored(score(ctx, z, None, k), z)
    ctx.check()


def test_largest_vocabulary(ctx):
    g = gen(3)
    for dtype in (torch.float32, torch.bfloat16):
        for rows in (1, 170):
            z = logits(g, rows, crf.abi.MAX_VOCAB, dtype)
            assert_scored(score(ctx, z, None, 32), z)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_and_alignment(ctx, dtype):
    g = gen(4)
    big = logits(g, 40, 3013, dtype)
    for first in range(9):
        z = big[:, first:first + 2900]
        t = torch.randint(0, 2900, (40,), device=DEV, generator=g, dtype=torch.int32)
        assert_scored(score(ctx, z, t, 5), z, t)
    z = big[::3, 1:2000]
    assert_scored(score(ctx, z, None, 5), z)
    # one row, whose stride says nothing
    assert_scored(score(ctx, big[7:8, :1234].as_strided((1, 1234), (0, 1)), None, 3), big[7:8, :1234])


def make_row(name, v, dtype):
    i = torch.arange(v, device=DEV, dtype=torch.float32)
    return {
        "rising": i / 64, "falling": -i / 64, "constant": torch.full_like(i, 2.5), "zeros of both signs": torch.where(i % 2 == 0, 0.0, -0.0),
        "one level in two": (i % 2) * 3, "steps": (i // 300) % 7, "sharp": torch.where(i == v - 2, 90.0, 0.0),
        "far down": i % 50 - 60000, "ruled out": torch.where(i % 97 == 5, i % 11, -math.inf), "all ruled out": torch.full_like(i, -math.inf),
        "one left": torch.where(i == v // 2, 1.0, -math.inf), "lowest values": torch.where(i % 3 == 0, torch.finfo(dtype).min, 1.0),
    }[name].to(dtype)[None]


ROWS = ["rising", "falling", "constant", "zeros of both signs", "one level in two", "steps", "sharp", "far down", "ruled out", "all ruled out",
        "one left", "lowest values"]


@pytest.mark.parametrize("name", ROWS)
@pytest.mark.parametrize("vocab", [300, 20000, 152064])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_ties_and_extremes(ctx, dtype, vocab, name):
    for rows in (1, 200):
        z = make_row(name, vocab, dtype).repeat(rows, 1)
        t = torch.arange(rows, device=DEV, dtype=torch.int32) * (vocab // (rows + 1))
        for k in (1, 17, 32):
            assert_scored(score(ctx, z, t, k), z, t)
    ctx.check()


def test_nan_and_infinity(ctx):
    g = gen(5)
    z = logits(g, 6, 5000, torch.float32)
    z[1, 77], z[2, 4999], z[3] = math.nan, math.inf, math.nan
    z[4, :4990] = math.nan
    out = score(ctx, z, torch.zeros(6, dtype=torch.int32, device=DEV), 12)
    for name in ("lse", "entropy", "logprob", "top_logprobs"):
        assert bool(out[name][1:5].isnan().all()), name
    assert_scored({k: v[[0, 5]] for k, v in out.items()}, z[[0, 5]], torch.zeros(2, dtype=torch.int32, device=DEV))
    ids = out["top_ids"].long().cpu()
    assert ids[2, 0] == 4999 and 77 not in ids[1].tolist() and ids[3].tolist() == list(range(12))
    last = sorted(range(4990, 5000), key=lambda i: -float(z[4, i]))
    assert ids[4].tolist() == last + [0, 1]


@pytest.mark.parametrize("rows,vocab", [(1, 40), (1, 300), (1, 5000), (400, 1030), (400, 5000), (400, 20000), (1, 152064), (310, 100000)])
def test_numbers_among_nan(ctx, rows, vocab):
    g = gen(13)
    for dtype in (torch.bfloat16, torch.float32):
        z = torch.full((rows, vocab), math.nan, device=DEV, dtype=dtype)
        ids = torch.randperm(vocab, device=DEV, generator=g)[:10]
        # of the ten, seven values in order and three -inf, which stand before NaN
        z[:, ids] = torch.tensor([7, 6, 5, 4, 3, 2, 1] + 3 * [-math.inf], device=DEV, dtype=dtype)
        want = ids[:7].tolist() + sorted(ids[7:].tolist())
        want += [i for i in range(vocab) if i not in want][:22]
        for k in (1, 9, 32):
            out = score(ctx, z, None, k)
            assert out["top_ids"].tolist() == [want[:k]] * rows and bool(out["lse"].isnan().all())


def test_targets_outside_the_vocabulary(ctx):
    g = gen(6)
    z = logits(g, 5, 700, torch.bfloat16)
    out = score(ctx, z, ints(3, 700, -2, -1, 2**31 - 1))
    with pytest.raises(CrfError, match="EINVAL"):
        ctx.check()
    assert_scored(out, z, ints(3, 0, 0, -1, 0))
    dz = torch.empty_like(z)
    ones = torch.ones(5, device=DEV)
    ctx.logprobs_grad(z, ints(3, 700, -2, -1, 2**31 - 1), out["lse"], dz, g_logprob=ones)
    with pytest.raises(CrfError, match="EINVAL"):
        ctx.check()
    assert_grad(dz, z, ints(3, 0, 0, -1, 0), out["lse"], ones)
    ctx.check()


def test_no_rows_and_single_outputs(ctx):
    g = gen(7)
    z = logits(g, 4, 999, torch.float32)
    ctx.logprobs(z[:0], lse=torch.empty(0, device=DEV))
    ctx.logprobs_grad(z[:0], None, torch.empty(0, device=DEV), z[:0])
    all_of = score(ctx, z, ints(1, 2, 3, 998), 6)
    for name in all_of:
        out = torch.full_like(all_of[name], 7)
        ctx.logprobs(z, ints(1, 2, 3, 998), **{name: out})
        assert torch.equal(out, all_of[name])
    ctx.logprobs(z)  # nothing wanted
    ctx.check()


# ---------------------------------------------------------------------------------------------- gradient
def assert_grad(dz, z, targets, lse, g=None, entropy=None, h=None):
    n, v = z.shape
    zero = torch.zeros(n, dtype=torch.float64, device=DEV)
    lse64 = lse.double()
    empty = lse == -math.inf
    l = z.double() - torch.where(empty, 0.0, lse64)[:, None]
    p = l.exp()
    gg = zero if g is None else torch.where(targets < 0, 0.0, g.double())
    hh, ent = (zero, zero) if h is None else (h.double(), entropy.double())
    lf = torch.where(p > 0, l, 0.0)
    want = -p * (gg[:, None] + hh[:, None] * (lf + ent[:, None]))
    by = gg.abs()[:, None] + hh.abs()[:, None] * (lf.abs() + ent.abs()[:, None])
    size = by * (p * (2.0**-21 + 2.0**-22 * (lf.abs() + lse64.abs().nan_to_num(posinf=0)[:, None])) + 2.0**-126)
    if g is not None:
        want.scatter_add_(1, targets.long().clamp(min=0)[:, None], gg[:, None])
        size.scatter_add_(1, targets.long().clamp(min=0)[:, None], 2.0**-23 * gg.abs()[:, None])
    want[empty] = 0
    t = torch.finfo(dz.dtype)
    tol = t.eps / 2 * want.abs().clamp(min=t.tiny) * 1.001 + size
    tol[empty] = 0
    worst = float(((dz.double() - want).abs() - tol).max())
    assert worst <= 0, worst


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 152064), (5, 257), (33, 5003), (3, 50001), (70000, 7), (40000, 33)])
def test_gradient(ctx, rows, vocab, dtype):
    g = gen(8)
    z = logits(g, rows, vocab, dtype)
    t = torch.randint(-1, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    a, b = normal(g, rows, dtype=torch.float32), normal(g, rows, dtype=torch.float32)
    out = score(ctx, z, t)
    for one, two in ((a, b), (a, None), (None, b), (None, None)):
        dz = torch.full_like(z, 7.0)
        ctx.logprobs_grad(z, None if one is None else t, out["lse"], dz, g_logprob=one, entropy=out["entropy"], g_entropy=two)
        assert_grad(dz, z, t, out["lse"], one, out["entropy"], two)
    ctx.logprobs_grad(z, t, out["lse"], z.copy_(z), g_logprob=a, entropy=out["entropy"], g_entropy=b)  # in place
    dz = torch.empty_like(z)
    assert not torch.equal(z, dz) or vocab == 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_strides_alignment_and_in_place(ctx, dtype):
    g = gen(9)
    big, other = logits(g, 30, 2011, dtype), logits(g, 30, 2027, dtype)
    for first, second, n in ((0, 0, 1999), (1, 1, 1800), (3, 2, 1900), (8, 16, 1777), (5, 13, 2000)):
        z, dz = big[:, first:first + n], other[:, second:second + n]
        t = torch.randint(0, n, (30,), device=DEV, generator=g, dtype=torch.int32)
        a, b = normal(g, 30, dtype=torch.float32), normal(g, 30, dtype=torch.float32)
        out, keep, keep_z = score(ctx, z, t), other.clone(), big.clone()
        ctx.logprobs_grad(z, t, out["lse"], dz, g_logprob=a, entropy=out["entropy"], g_entropy=b)
        assert_grad(dz, z, t, out["lse"], a, out["entropy"], b)
        got = dz.clone()
        dz.copy_(keep[:, second:second + n])
        assert torch.equal(other, keep) and torch.equal(big, keep_z)  # nothing outside was written
        ctx.logprobs_grad(z, t, out["lse"], z, g_logprob=a, entropy=out["entropy"], g_entropy=b)
        assert torch.equal(z, got)
        z.copy_(keep_z[:, first:first + n])
        assert torch.equal(big, keep_z)


@pytest.mark.parametrize("name", ROWS)
def test_gradient_of_extremes(ctx, name):
    z = make_row(name, 5003, torch.float32).repeat(3, 1)
    t, a, b = ints(5, 2501, -1), torch.tensor([1.0, -2.0, 3.0], device=DEV), torch.tensor([0.5, 0.0, -1.0], device=DEV)
    out = score(ctx, z, t)
    dz = torch.empty_like(z)
    ctx.logprobs_grad(z, t, out["lse"], dz, g_logprob=a, entropy=out["entropy"], g_entropy=b)
    assert_grad(dz, z, t, out["lse"], a, out["entropy"], b)
    assert bool(dz.isfinite().all())


def test_gradient_is_that_of_the_formula_and_of_differences(ctx):
    g = gen(10)
    z, t = logits(g, 3, 301, torch.float32, wide=1.0), ints(7, 300, 0)
    a, b = normal(g, 3, dtype=torch.float32), normal(g, 3, dtype=torch.float32)
    out, dz = score(ctx, z, t), torch.empty_like(z)
    ctx.logprobs_grad(z, t, out["lse"], dz, g_logprob=a, entropy=out["entropy"], g_entropy=b)

    def loss(x):
        l = torch.log_softmax(x, 1)
        return (l.gather(1, t.long()[:, None])[:, 0] * a.double()).sum() - ((l.exp() * l).sum(1) * b.double()).sum()

    leaf = z.double().requires_grad_()
    want = torch.autograd.grad(loss(leaf), leaf)[0]
    # the formula's own lse and entropy are off the given ones by 2^-16 (1 + W), W < 8, each in units of p (|g| + |h| (|l| + |H|))
    assert bool(((dz.double() - want).abs() <= 2.0**-12 * (want.abs() + 0.1)).all())
    e, step = normal(g, 3, 301, dtype=torch.float32), 2.0**-6
    sides, exact = [], []
    for s in (step, -step):
        got = score(ctx, z + s * e, t)
        sides.append(float((got["logprob"].double() * a.double()).sum() + (got["entropy"].double() * b.double()).sum()))
        exact.append(float(loss((z + s * e).double())))
    off = abs((exact[0] - exact[1]) / (2 * step) - float((want * e.double()).sum()))
    # six numbers a side, each off by 2^-15 (1 + W) at most, times |g| or |h| < 4; the gradient itself by the bound above
    room = 2 * 6 * 4 * 9 * 2.0**-15 / (2 * step) + 2.0**-12 * float(((want.abs() + 0.1) * e.double().abs()).sum())
    assert abs((sides[0] - sides[1]) / (2 * step) - float((dz.double() * e.double()).sum())) <= off + room


def test_scores_repeat_their_bits_on_streams_and_in_graphs(ctx):
    g = gen(11)
    for rows in (2, 300):
        z = logits(g, rows, 40003, torch.bfloat16)
        t = torch.randint(0, 40003, (rows,), device=DEV, generator=g, dtype=torch.int32)
        first = score(ctx, z, t, 20)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        second = {k: torch.empty_like(v) for k, v in first.items()}
        side.wait_stream(torch.cuda.current_stream())
        ctx.logprobs(z, t, stream=side, **second)
        side.synchronize()
        third, dz = {k: torch.empty_like(v) for k, v in first.items()}, torch.empty_like(z)
        graph = torch.cuda.CUDAGraph()
        ones = torch.ones(rows, device=DEV)
        with torch.cuda.graph(graph):
            ctx.logprobs(z, t, **third)
            ctx.logprobs_grad(z, t, third["lse"], dz, g_logprob=ones)
        for _ in range(2):
            for v in third.values():
                v.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for k in first:
            assert torch.equal(first[k], second[k]) and torch.equal(first[k], third[k])
        assert_grad(dz, z, t, third["lse"], ones)


def test_rows_behind_2_31_elements(ctx):
    rows = 2**31 // 152064 + 2
    z = torch.zeros(rows, 152064, dtype=torch.bfloat16, device=DEV)
    g = gen(12)
    z[-2:] = logits(g, 2, 152064, torch.bfloat16)
    t = torch.full((rows,), 3, dtype=torch.int32, device=DEV)
    out = score(ctx, z, t, 2)
    last = {k: v[-2:] for k, v in out.items()}
    assert_scored(last, z[-2:], t[-2:])
    ones, keep = torch.ones(rows, device=DEV), z[-2:].clone()
    ctx.logprobs_grad(z, t, out["lse"], z, g_logprob=ones)
    assert_grad(z[-2:], keep, t[-2:], last["lse"], ones[-2:])
