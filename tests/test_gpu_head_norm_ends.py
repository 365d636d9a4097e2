"""The gradient of normed heads whose tensors end where their memory does, or whose heads lie far apart: threads that have no head read nothing
(what they would have read was no part of any result, but could lie outside every allocation)."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads_outside", [False, True])
@pytest.mark.parametrize("rows,hq,hk,dim,rot", [(1, 1, 1, 128, 128), (44, 4, 2, 96, 96), (20, 28, 7, 128, 64), (3, 40, 8, 128, 128), (643, 12, 2, 64, 64),
                                               (650, 9, 5, 128, 128), (4001, 3, 0, 64, 32)])
def test_gradient_at_the_ends_of_memory(ctx, rows, hq, hk, dim, rot, heads_outside, dtype):
    g = gen(41)
    a = dict(theta=1e4, rot_dim=rot)
    rope = crf.Rope(dim, **a)

    def tensor(heads):
        # heads outside: a head behind the last one is rows x dim elements further on
        t = normal(g, heads, rows, dim, dtype=dtype).transpose(0, 1) if heads_outside else normal(g, rows, heads, dim, dtype=dtype)
        return t

    pos = torch.randint(0, 9000, (rows,), device=DEV, generator=g, dtype=torch.int32)
    x, grad, dx, w, dgain = tensor(hq), tensor(hq), tensor(hq), gain_of(g, dim, dtype), torch.empty(dim, device=DEV)
    more = {}
    if hk:
        k, k_grad, k_dx, k_w, k_dgain = tensor(hk), tensor(hk), tensor(hk), gain_of(g, dim, dtype), torch.empty(dim, device=DEV)
        more = dict(k=k, k_gain=k_w, k_grad=k_grad, k_dx=k_dx, k_dgain=k_dgain)
    ctx.norm_rotary_grad(rope, pos, x, w, grad, dx, dgain, ctx.norm_rotary_workspace(rope, rows), eps=EPS, **more)
    assert_grads(dx, dgain, x, w, grad, pos, dim, a)
    if hk:
        assert_grads(k_dx, k_dgain, k, k_w, k_grad, pos, dim, a)
    ctx.check()
