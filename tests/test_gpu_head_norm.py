"""Norms of query and key heads with the position rotation, their gradient and the append of normed heads, against 64-bit
formulas.

Tolerances count roundings. Forward: half a step of the type relative to the value, and 2^-19 of |u| + |v|, the pair before it
is turned (the sum of at most 256 squares adds under 32 roundings to the mean square, half as many relative to its root; the
reciprocal root is off by 2^-22; angle, sine, cosine and products 2^-21 as without a norm). Gradient of x: the same and 2^-18
of r (|v| + |x| r^2 mean |v x|), whose two terms carry those roundings and the sum's. Gradient of the gain: no thread, block or
final sum of these tests adds over 512 terms in a row, so 2^-15 of the sum of the terms' sizes."""
import math

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300.abi import CrfError
from tests.test_gpu_extend import DEV, PAGE, ROPES, gen, ints, normal, pages_for, rotate64, tables_of

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


def gain_of(g, dim, dtype):
    return (1 + 0.2 * normal(g, dim, dtype=torch.float32)).to(dtype)


def norm64(x, gain, eps=EPS):
    x = x.double()
    return x * (x.square().mean(-1, keepdim=True) + eps).rsqrt() * gain.double()


def assert_normed(got, x, gain, pos, dim, a, eps=EPS):
    n = norm64(x, gain, eps)
    want, size = rotate64(n, pos, dim, a)
    size = torch.maximum(size, n.abs())
    t = torch.finfo(got.dtype)
    tol = t.eps / 2 * want.abs().clamp(min=t.tiny) * 1.001 + 2.0**-19 * size
    worst = float(((got.double() - want).abs() - tol).max())
    assert worst <= 0, worst


def grads64(x, gain, grad, pos, dim, a, eps=EPS):
    """(dx, its roundings' size, dgain, its terms' size) in 64 bits."""
    u, size_u = rotate64(grad, pos, dim, a, inverse=True)
    size_u = torch.maximum(size_u, grad.double().abs())
    x, w = x.double(), gain.double()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    v, size_v = u * w, size_u * w.abs()
    dx = r * (v - x * r.square() * (v * x).mean(-1, keepdim=True))
    size = r * (size_v + x.abs() * r.square() * (size_v * x.abs()).mean(-1, keepdim=True))
    return dx, size, (u * x * r).sum((0, 1)), (size_u * (x * r).abs()).sum((0, 1))


def assert_grads(dx, dgain, x, gain, grad, pos, dim, a, eps=EPS):
    want, size, want_gain, size_gain = grads64(x, gain, grad, pos, dim, a, eps)
    t = torch.finfo(dx.dtype)
    tol = t.eps / 2 * want.abs().clamp(min=t.tiny) * 1.001 + 2.0**-18 * size
    worst = float(((dx.double() - want).abs() - tol).max())
    assert worst <= 0, worst
    worst = float(((dgain.double() - want_gain).abs() - 2.0**-15 * size_gain).max())
    assert worst <= 0, worst


SHAPES = ((1, 4, 2, 64), (37, 28, 4, 128), (700, 3, 1, 64), (650, 9, 5, 128))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("name", sorted(ROPES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_norm_of_types_layouts_and_scalings(ctx, dtype, name, layout):
    a = dict(ROPES[name], layout=layout)
    g = gen(1)
    for rows, hq, hk, dim in SHAPES:
        x = normal(g, rows, hq + hk, dim, dtype=dtype) * 3
        grad = normal(g, rows, hq + hk, dim, dtype=dtype)
        gq, gk = gain_of(g, dim, dtype), gain_of(g, dim, dtype)
        pos = torch.randint(0, 131072, (rows,), device=DEV, generator=g, dtype=torch.int32)
        q, k = torch.empty(rows, hq, dim, dtype=dtype, device=DEV), torch.empty(rows, hk, dim, dtype=dtype, device=DEV)
        rope = crf.Rope(dim, **a)
        ctx.norm_rotary(rope, pos, x[:, :hq], gq, out=q, k=x[:, hq:], k_gain=gk, k_out=k, eps=EPS)
        assert_normed(q, x[:, :hq], gq, pos, dim, a)
        assert_normed(k, x[:, hq:], gk, pos, dim, a)
        dgq, dgk = torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
        ctx.norm_rotary_grad(rope, pos, x[:, :hq], gq, grad[:, :hq], q, dgq, ctx.norm_rotary_workspace(rope, rows), k=x[:, hq:],
                             k_gain=gk, k_grad=grad[:, hq:], k_dx=k, k_dgain=dgk, eps=EPS)
        assert_grads(q, dgq, x[:, :hq], gq, grad[:, :hq], pos, dim, a)
        assert_grads(k, dgk, x[:, hq:], gk, grad[:, hq:], pos, dim, a)
    ctx.check()


@pytest.mark.parametrize("dim,rot", [(2, 2), (6, 4), (80, 40), (96, 96), (256, 256), (256, 2), (66, 66), (64, 20), (8, 8), (256, 16), (24, 16)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_of_odd_heads(ctx, dtype, dim, rot, layout):
    g = gen(2)
    a = dict(theta=1e4, rot_dim=rot, layout=layout)
    rope = crf.Rope(dim, **a)
    for rows, heads in ((1, 1), (19, 5), (613, 2)):
        x, grad, w = normal(g, rows, heads, dim, dtype=dtype), normal(g, rows, heads, dim, dtype=dtype), gain_of(g, dim, dtype)
        pos = torch.randint(0, 5000, (rows,), device=DEV, generator=g, dtype=torch.int32)
        out, dgain = torch.empty_like(x), torch.empty(dim, device=DEV)
        ctx.norm_rotary(rope, pos, x, w, out=out, eps=EPS)
        assert_normed(out, x, w, pos, dim, a)
        ctx.norm_rotary_grad(rope, pos, x, w, grad, out, dgain, ctx.norm_rotary_workspace(rope, rows), eps=EPS)
        assert_grads(out, dgain, x, w, grad, pos, dim, a)
    ctx.check()


def test_norm_of_many_heads(ctx):
    # more heads than a row's blocks take side by side in the gradient, and than a block has slots
    g = gen(3)
    a = dict(theta=1e4)
    rope = crf.Rope(64, **a)
    for heads in (130, 700):
        x, grad, w = normal(g, 5, heads, 64), normal(g, 5, heads, 64), gain_of(g, 64, torch.bfloat16)
        k, kg = normal(g, 5, 3, 64), normal(g, 5, 3, 64)
        pos = ints(0, 3, 100, 7, 70000)
        out, ko, dgain, kdgain = torch.empty_like(x), torch.empty_like(k), torch.empty(64, device=DEV), torch.empty(64, device=DEV)
        ctx.norm_rotary(rope, pos, x, w, out=out, k=k, k_gain=w, k_out=ko, eps=EPS)
        assert_normed(out, x, w, pos, 64, a)
        assert_normed(ko, k, w, pos, 64, a)
        ctx.norm_rotary_grad(rope, pos, x, w, grad, out, dgain, ctx.norm_rotary_workspace(rope, 5), k=k, k_gain=w, k_grad=kg, k_dx=ko,
                             k_dgain=kdgain, eps=EPS)
        assert_grads(out, dgain, x, w, grad, pos, 64, a)
        assert_grads(ko, kdgain, k, w, kg, pos, 64, a)
    ctx.check()


def test_norm_strides_alignment_and_in_place(ctx):
    g = gen(4)
    a = dict(theta=1e4)
    rope = crf.Rope(64, **a)
    w = gain_of(g, 64, torch.bfloat16)
    odd = torch.cat((w[:1], w))[1:]  # the same gain, two bytes off a 16-byte boundary
    big, wide = normal(g, 11, 9, 72), normal(g, 11, 9, 72)
    for pick in (lambda t: t[:, 2:7, 3:67], lambda t: t[:, :, 8:72], lambda t: t.transpose(0, 1)[..., :64]):
        view, grad = pick(big), pick(wide)
        pos = ints(*range(100, 100 + len(view)))
        keep, keep_wide, x = big.clone(), wide.clone(), view.clone()
        for gain in (w, odd):
            ctx.norm_rotary(rope, pos, view, gain, eps=EPS)  # in place
            assert_normed(view, x, w, pos, 64, a)
            view.copy_(x)
            assert torch.equal(big, keep)  # nothing outside the view was touched
            dgain, ws = torch.empty(64, device=DEV), ctx.norm_rotary_workspace(rope, len(view))
            g0 = grad.clone()
            ctx.norm_rotary_grad(rope, pos, view, gain, grad, view, dgain, ws, eps=EPS)  # over x
            assert_grads(view, dgain, x, w, g0, pos, 64, a)
            view.copy_(x)
            ctx.norm_rotary_grad(rope, pos, view, gain, grad, grad, dgain, ws, eps=EPS)  # over the gradient
            assert_grads(grad, dgain, x, w, g0, pos, 64, a)
            grad.copy_(g0)
            assert torch.equal(big, keep) and torch.equal(wide, keep_wide)


def test_norm_of_broadcast_heads(ctx):
    # strides of 0 in what is read: one row for all positions, one gradient for all heads
    g = gen(5)
    a = dict(theta=1e4)
    rope = crf.Rope(128, **a)
    x, grad, w = normal(g, 1, 6, 128).expand(40, 6, 128), normal(g, 40, 1, 128).expand(40, 6, 128), gain_of(g, 128, torch.bfloat16)
    pos = ints(*range(40))
    out, dgain = torch.empty(40, 6, 128, dtype=torch.bfloat16, device=DEV), torch.empty(128, device=DEV)
    ctx.norm_rotary(rope, pos, x, w, out=out, eps=EPS)
    assert_normed(out, x, w, pos, 128, a)
    ctx.norm_rotary_grad(rope, pos, x, w, grad, out, dgain, ctx.norm_rotary_workspace(rope, 40), eps=EPS)
    assert_grads(out, dgain, x, w, grad, pos, 128, a)


def test_norm_of_zeros_and_of_small_and_large_values(ctx):
    g = gen(6)
    a = dict(theta=1e4)
    rope = crf.Rope(128, **a)
    w = gain_of(g, 128, torch.float32)
    x = normal(g, 6, 2, 128, dtype=torch.float32)
    x *= torch.tensor([0.0, 1e-18, 1e-4, 1.0, 1e6, 1e17], device=DEV)[:, None, None]
    grad, pos = normal(g, 6, 2, 128, dtype=torch.float32), ints(0, 1, 2, 3, 4, 5)
    out, dgain = torch.empty_like(x), torch.empty(128, device=DEV)
    for eps in (1e-6, 1e-2):
        ctx.norm_rotary(rope, pos, x, w, out=out, eps=eps)
        # eps is a rounded number: so is the root where it decides
        assert_normed(out, x, w, pos, 128, a, eps=float(torch.tensor(eps)))
        assert not out[0].any()
        ctx.norm_rotary_grad(rope, pos, x, w, grad, out, dgain, ctx.norm_rotary_workspace(rope, 6), eps=eps)
        assert_grads(out, dgain, x, w, grad, pos, 128, a, eps=float(torch.tensor(eps)))
    ctx.norm_rotary(rope, pos[2:], x[2:], w, out=out[2:], eps=0.0)
    assert_normed(out[2:], x[2:], w, pos[2:], 128, a, eps=0.0)


def test_norm_of_no_rows(ctx):
    rope = crf.Rope(64)
    x, w = torch.empty(0, 4, 64, device=DEV), torch.ones(64, device=DEV)
    ctx.norm_rotary(rope, ints(), x, w)
    dgain = torch.full((64,), 7.0, device=DEV)
    ctx.norm_rotary_grad(rope, ints(), x, w, x, x, dgain, ctx.norm_rotary_workspace(rope, 0))
    assert not dgain.any()
    ctx.check()


def test_norm_gradient_is_that_of_the_formula_and_of_differences(ctx):
    g = gen(7)
    a = dict(theta=1e4, rot_dim=32, scaling="bands", factor=4.0, low=1.0, high=16.0, original=512, magnitude=1.2)
    rope = crf.Rope(64, **a)
    x, grad, w = (normal(g, 9, 3, 64, dtype=torch.float32) for _ in range(3))
    w = gain_of(g, 64, torch.float32)
    pos = torch.randint(0, 4000, (9,), device=DEV, generator=g, dtype=torch.int32)
    dx, dgain = torch.empty_like(x), torch.empty(64, device=DEV)
    ctx.norm_rotary_grad(rope, pos, x, w, grad, dx, dgain, ctx.norm_rotary_workspace(rope, 9), eps=EPS)
    lx, lw = x.double().requires_grad_(), w.double().requires_grad_()
    loss = lambda t, v: (rotate64(norm64(t, v), pos, 64, a)[0] * grad.double()).sum()  # noqa: E731
    want_x, want_w = torch.autograd.grad(loss(lx, lw), (lx, lw))
    _, size, _, size_gain = grads64(x, w, grad, pos, 64, a)
    assert bool(((dx.double() - want_x).abs() <= 2.0**-24 * want_x.abs() + 2.0**-18 * size).all())
    assert bool(((dgain.double() - want_w).abs() <= 2.0**-15 * size_gain).all())
    # differences of the call itself, along one direction of x and one of the gain, against the gradients that it gave: off
    # by what differences of the 64-bit formula are off, and by 1728 outputs of at most 2^-19 (|u| + |v|) each
    step = 2.0**-5
    for t, is_x in ((normal(g, 9, 3, 64, dtype=torch.float32), True), (normal(g, 64, dtype=torch.float32), False)):
        sides, exact, room = [], [], 0.0
        for s in (step, -step):
            xs, ws = (x + s * t, w) if is_x else (x, w + s * t)
            y = torch.empty_like(x)
            ctx.norm_rotary(rope, pos, xs, ws, out=y, eps=EPS)
            sides.append(float((y.double() * grad.double()).sum()))
            exact.append(float(loss(xs.double(), ws.double())))
            room += float((2.0**-18 * rotate64(norm64(xs, ws), pos, 64, a)[1].clamp(min=1.0) * grad.double().abs()).sum())
        got = (sides[0] - sides[1]) / (2 * step)
        slope = float((dx.double() * t.double()).sum()) if is_x else float((dgain.double() * t.double()).sum())
        wanted = float((want_x * t.double()).sum()) if is_x else float((want_w * t.double()).sum())
        off = abs((exact[0] - exact[1]) / (2 * step) - wanted)
        assert abs(got - slope) <= off + room / (2 * step) + 2.0**-15 * float(size_gain.sum())


@pytest.mark.parametrize("name,layout", [("whole", "half"), ("bands", "half"), ("part", "interleaved")])
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (28, 4, 128), (3, 3, 64)])
@pytest.mark.parametrize("with_q", [True, False])
def test_append_of_normed_heads_writes_its_slots_only(ctx, hq, hkv, dim, name, layout, with_q):
    g = gen(8)
    new, pos = [1, 40, 0, 17, 1], [0, 31, 5, 16, 777]
    tables, total = tables_of(g, [pages_for(m + p) for m, p in zip(new, pos)])
    kp, vp = normal(g, total, hkv, PAGE, dim), normal(g, total, hkv, PAGE, dim)
    kp0, vp0 = kp.clone(), vp.clone()
    rows = sum(new)
    qkv = normal(g, rows, hq + 2 * hkv, dim) * 2
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    gq, gk = gain_of(g, dim, torch.bfloat16), gain_of(g, dim, torch.bfloat16)
    at = torch.cat([torch.arange(p, p + m) for m, p in zip(new, pos)]).to(DEV)
    req = torch.cat([torch.full((m,), i) for i, m in enumerate(new)])
    page = torch.stack([tables[i][p // PAGE] for i, p in zip(req.tolist(), at.tolist())]).long()
    a = dict(ROPES[name], layout=layout)
    q_out = torch.empty(rows, hq, dim, dtype=torch.bfloat16, device=DEV)
    pool = crf.KVPool([torch.zeros_like(kp), kp], [torch.zeros_like(vp), vp])
    more = dict(q=q, q_out=q_out, q_gain=gq) if with_q else {}
    ctx.cache_append(pool, 1, crf.Chunks(tables, new, pos), k, v, rope=crf.Rope(dim, **a), k_gain=gk, eps=EPS, **more)
    ctx.check()
    assert_normed(kp[page, :, at % PAGE], k, gk, at, dim, a)
    if with_q:
        assert_normed(q_out, q, gq, at, dim, a)
    assert torch.equal(vp[page, :, at % PAGE], v)
    kp[page, :, at % PAGE] = kp0[page, :, at % PAGE]
    vp[page, :, at % PAGE] = vp0[page, :, at % PAGE]
    assert torch.equal(kp, kp0) and torch.equal(vp, vp0)
    assert not pool.k_pages[0].any() and not pool.v_pages[0].any()


@pytest.mark.parametrize("off", [0, 1])
def test_append_of_normed_heads_leaves_out_pages_outside_the_pool(ctx, off):
    g = gen(9)
    kp, vp = normal(g, 4, 2, PAGE, 64), normal(g, 4, 2, PAGE, 64)
    kp0, vp0 = kp.clone(), vp.clone()
    # `off`: heads that start between 16-byte boundaries take the form of a warp a head
    k, v = normal(g, 20, 2, 72)[..., off:off + 64], normal(g, 20, 2, 64)
    w, pool = gain_of(g, 64, torch.bfloat16), crf.KVPool([kp], [vp])
    for bad in (4, -1, 2**31 - 1, -(2**31)):
        ctx.cache_append(pool, 0, crf.Chunks([ints(2, bad)], [20], [0]), k, v, rope=crf.Rope(64), k_gain=w, eps=EPS)
        with pytest.raises(CrfError, match="EINVAL"):
            ctx.check()
        assert_normed(kp[2].transpose(0, 1), k[:16], w, ints(*range(16)), 64, dict(theta=1e4))
        assert torch.equal(vp[2].transpose(0, 1), v[:16])
        kp[2], vp[2] = kp0[2], vp0[2]
        assert torch.equal(kp, kp0) and torch.equal(vp, vp0)
    ctx.check()


def test_norm_repeats_its_bits_on_streams_and_in_graphs(ctx):
    g = gen(10)
    rope = crf.Rope(128, theta=1e6)
    x, grad, w = normal(g, 1500, 7, 128), normal(g, 1500, 7, 128), gain_of(g, 128, torch.bfloat16)
    pos = torch.randint(0, 9000, (1500,), device=DEV, generator=g, dtype=torch.int32)

    def call(out, dx, dgain, ws, stream=None):
        ctx.norm_rotary(rope, pos, x, w, out=out, eps=EPS, stream=stream)
        ctx.norm_rotary_grad(rope, pos, x, w, grad, dx, dgain, ws, eps=EPS, stream=stream)

    buffers = lambda: (torch.empty_like(x), torch.empty_like(x), torch.empty(128, device=DEV), ctx.norm_rotary_workspace(rope, 1500))  # noqa: E731
    first, second, third = buffers(), buffers(), buffers()
    call(*first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(*second, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*third)
    for _ in range(2):
        for t in third:
            t.zero_()
        graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first[:3], second, third):
        assert torch.equal(a, b) and torch.equal(a, c)
    x.neg_()  # a replay reads what is there then
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(third[0], -first[0])


def test_norm_rows_behind_others_far_apart(ctx):
    # rows whose places differ by more than 2^31 elements
    big = torch.empty(2**31 + 4096, dtype=torch.bfloat16, device=DEV)
    x = big.as_strided((2, 2, 128), (2**31, 128, 1))
    g = gen(11)
    x.copy_(normal(g, 2, 2, 128))
    w, pos = gain_of(g, 128, torch.bfloat16), ints(5, 6)
    keep, dgain = x.clone(), torch.empty(128, device=DEV)
    a = dict(theta=1e4)
    rope, grad = crf.Rope(128, **a), normal(g, 2, 2, 128)
    dx = torch.empty_like(keep)
    ctx.norm_rotary_grad(rope, pos, x, w, grad, dx, dgain, ctx.norm_rotary_workspace(rope, 2), eps=EPS)
    assert_grads(dx, dgain, keep, w, grad, pos, 128, a)
    ctx.norm_rotary(rope, pos, x, w, eps=EPS)
    assert_normed(x, keep, w, pos, 128, a)
    assert math.isfinite(float(dgain.sum()))
