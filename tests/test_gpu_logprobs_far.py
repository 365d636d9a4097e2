"""Log probabilities of logits far from zero: the maximum is taken off first, so they are as exact there as around zero.

Two bounds. (a) Logits that are shifted without a rounding have the same differences from their maximum, and so bit for bit the
same log probabilities and entropies. (b) Against 64 bits, the tolerance of test_gpu_logprobs.py without its parts in |lse| and
|z|: the sum's 2^-16 (1 + W), W = sum p |z - max|, and three roundings of the two differences and the logarithm, 2^-22 (|z - max| + log s)."""
import math

import pytest
import torch

import paper_2609_30884_gb300 as crf
from tests.test_gpu_extend import DEV, gen, normal
from tests.test_gpu_logprobs import score

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


# rows of a warp each, of a cluster, of a block
SIZES = [(3, 500), (2600, 3001), (2, 40003), (700, 20011), (1, 152064)]


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype,step,limit,shifts", [(torch.float32, 2.0**-8, 12, (2.0**7, -(2.0**7), 2.0**14, -(2.0**14))),
                                                    (torch.float16, 2.0**-3, 12, (2.0**7, -(2.0**7))), (torch.bfloat16, 1.0, 20, (2.0**7, -(2.0**7)))])
def test_shifted_logits_have_the_same_log_probabilities(ctx, dtype, step, limit, shifts, rows, vocab):
    g = gen(1)
    # multiples of `step` up to `limit`, so that a shift by a power of two rounds none of them
    z = ((normal(g, rows, vocab, dtype=torch.float32) * 3).clamp(-limit, limit) / step).round() * step
    t = torch.randint(0, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    want = score(ctx, z.to(dtype), t, 20)
    for shift in shifts:
        moved = (z + shift).to(dtype)
        assert torch.equal(moved.double(), z.double() + shift)
        got = score(ctx, moved, t, 20)
        for name in ("logprob", "top_logprobs", "top_ids", "entropy"):
            assert torch.equal(got[name], want[name]), (name, shift)


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_log_probabilities_of_far_logits(ctx, dtype, rows, vocab):
    g = gen(2)
    for shift in (0.0, 30.0, -300.0, 3000.0, -60000.0, 1e6):
        z = (normal(g, rows, vocab, dtype=torch.float32) * 3 + shift).to(dtype)
        t = torch.randint(0, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
        out = score(ctx, z, t, 8)
        x = z.double()
        x -= x.amax(1, keepdim=True)
        e = x.exp()
        s = e.sum(1, keepdim=True)
        w = (e / s * x.abs()).sum(1, keepdim=True)
        for got, ids in ((out["logprob"][:, None], t.long()[:, None]), (out["top_logprobs"], out["top_ids"].long())):
            want = x.gather(1, ids) - s.log()
            tol = 2.0**-16 * (1 + w) + 2.0**-22 * (x.gather(1, ids).abs() + s.log())
            assert bool(((got.double() - want).abs() <= tol).all()), (shift, float(((got.double() - want).abs() - tol).max()))


@pytest.mark.parametrize("vocab", [300, 30000])
def test_rows_without_log_probabilities(ctx, vocab):
    # nothing but ruled-out tokens, one number among them, NaN, +inf: as around zero
    z = torch.full((4, vocab), -math.inf, device=DEV)
    z[1, 7], z[2, 9], z[3, 9] = -60000.0, math.nan, math.inf
    for rows in (4, 1):
        out = score(ctx, z[:rows], torch.full((rows,), 7, dtype=torch.int32, device=DEV), 2)
        assert out["logprob"][0] == -math.inf and bool((out["top_logprobs"][0] == -math.inf).all())
    out = score(ctx, z, torch.full((4,), 7, dtype=torch.int32, device=DEV), 2)
    assert out["logprob"][1] == 0 and out["top_logprobs"][1].tolist() == [0, -math.inf] and out["top_ids"][1, 0] == 7
    assert bool(out["logprob"][2:].isnan().all()) and bool(out["top_logprobs"][2:].isnan().all())
