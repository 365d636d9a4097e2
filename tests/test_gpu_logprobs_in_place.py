"""The gradient of log probabilities written over the logits: bit for bit what the call gives elsewhere, at every size, type and alignment
(test_gradient of test_gpu_logprobs.py makes the call and compares what it wrote with memory that nothing has written)."""
import pytest
import torch

import paper_2609_30884_gb300 as crf
from tests.test_gpu_extend import DEV, gen, normal
from tests.test_gpu_logprobs import assert_grad, logits, score

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 152064), (5, 257), (33, 5003), (3, 50001), (70000, 7), (40000, 33), (2, 1 << 20)])
@pytest.mark.parametrize("spare", [0, 3])
def test_gradient_in_place(ctx, rows, vocab, dtype, spare):
    g = gen(31)
    # rows of a buffer with `spare` entries at each end, which stay as they are
    big = logits(g, rows, vocab + 2 * spare, dtype)
    z = big[:, spare:spare + vocab]
    keep = big.clone()
    t = torch.randint(-1, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    a, b = normal(g, rows, dtype=torch.float32), normal(g, rows, dtype=torch.float32)
    out = score(ctx, z, t)
    for one, two in ((a, b), (a, None), (None, b), (None, None)):
        kw = dict(g_logprob=one, entropy=out["entropy"], g_entropy=two)
        dz = torch.full_like(big, 7.0)[:, spare:spare + vocab]
        ctx.logprobs_grad(z, None if one is None else t, out["lse"], dz, **kw)
        assert torch.equal(big, keep)
        assert_grad(dz, z, t, out["lse"], one, out["entropy"], two)
        ctx.logprobs_grad(z, None if one is None else t, out["lse"], z, **kw)
        assert torch.equal(z, dz)
        z.copy_(keep[:, spare:spare + vocab])
        assert torch.equal(big, keep)
    ctx.check()
