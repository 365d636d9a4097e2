"""The gradient of normed heads where its blocks walk many tiles of rows: angles change buffers, positions are refilled, and a block's last
batch and last tile are not full. Formulas and tolerances are those of test_gpu_head_norm.py (a thread adds at most 110 terms of the
gain's gradient, a block 64, the last sums 50)."""
import pytest
import torch

import paper_2609_30884_gb300 as crf
from tests.test_gpu_extend import DEV, gen, normal
from tests.test_gpu_head_norm import EPS, assert_grads, gain_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


# rows, heads of x and k, head_dim, elements that turn. With 152 SMs, for 16-bit half-layout heads: tiles a block, and of a batch
SHAPES = [
    (16387, 28, 4, 128, 128),   # 54, 8
    (4099, 9, 5, 128, 64),      # 13, 8
    (90011, 3, 1, 64, 64),      # 18, 4 (of 8 rows)
    (100003, 1, 1, 64, 64),     # 10, 2 (of 16)
    (250007, 1, 0, 32, 32),     # 6, 1 (of 32)
    (61001, 2, 1, 64, 32),      # 20, 8 (of 4)
    (9001, 5, 2, 256, 256),     # 14, 8; fp32 interleaved heads of 256 a warp each, 15 rows a block
    (9001, 3, 2, 80, 40),       # odd heads: a warp each where pieces are no 16 bytes
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,hq,hk,dim,rot", SHAPES)
def test_gradient_over_many_tiles(ctx, rows, hq, hk, dim, rot, dtype, layout):
    g = gen(21)
    a = dict(theta=1e6, rot_dim=rot, layout=layout)
    x = normal(g, rows, hq + hk, dim, dtype=dtype)
    grad = normal(g, rows, hq + hk, dim, dtype=dtype)
    gq, gk = gain_of(g, dim, dtype), gain_of(g, dim, dtype)
    # positions that no row shares with its neighbours, or with the row a batch, a tile or a block's turn away
    pos = torch.randperm(1 << 18, device=DEV, generator=g)[:rows].to(torch.int32)
    rope, ws = crf.Rope(dim, **a), ctx.norm_rotary_workspace(crf.Rope(dim, **a), rows)

    def call(dx, dgq, dgk):
        k = dict(k=x[:, hq:], k_gain=gk, k_grad=grad[:, hq:], k_dx=dx[:, hq:], k_dgain=dgk) if hk else {}
        ctx.norm_rotary_grad(rope, pos, x[:, :hq], gq, grad[:, :hq], dx[:, :hq], dgq, ws, eps=EPS, **k)

    dx, dgq, dgk = torch.empty_like(x), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    call(dx, dgq, dgk)
    assert_grads(dx[:, :hq], dgq, x[:, :hq], gq, grad[:, :hq], pos, dim, a)
    if hk:
        assert_grads(dx[:, hq:], dgk, x[:, hq:], gk, grad[:, hq:], pos, dim, a)
    # the same bits again, over x and over the gradient
    for over in (x, grad):
        keep, again = over.clone(), (torch.empty_like(dgq), torch.empty_like(dgk))
        call(over, *again)
        assert torch.equal(over, dx) and torch.equal(again[0], dgq) and (not hk or torch.equal(again[1], dgk))
        over.copy_(keep)
    ctx.check()


def test_gradient_over_many_tiles_in_a_graph(ctx):
    # replayed over other positions and values than it was captured with
    g = gen(22)
    rows, dim, a = 5003, 128, dict(theta=1e6)
    rope, w = crf.Rope(dim, **a), gain_of(g, dim, torch.bfloat16)
    x, grad = normal(g, rows, 7, dim), normal(g, rows, 7, dim)
    pos = torch.randint(0, 9000, (rows,), device=DEV, generator=g, dtype=torch.int32)
    dx, dgain, ws = torch.empty_like(x), torch.empty(dim, device=DEV), ctx.norm_rotary_workspace(rope, rows)
    ctx.norm_rotary_grad(rope, pos, x, w, grad, dx, dgain, ws, eps=EPS)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.norm_rotary_grad(rope, pos, x, w, grad, dx, dgain, ws, eps=EPS)
    for _ in range(3):
        x.normal_(generator=g), grad.normal_(generator=g), pos.random_(0, 131072, generator=g)
        graph.replay()
        torch.cuda.synchronize()
        assert_grads(dx, dgain, x, w, grad, pos, dim, a)
    ctx.check()
