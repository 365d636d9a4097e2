"""Attention over so many keys that one CTA's sums run over thousands of tiles.

A cache that repeats a few pages R times has every score R times: o is that of the pages alone, lse is larger by log R. So
the 64-bit formula is needed over the few keys only, whatever the length. Tolerances are those of test_gpu_extend.py
(roundings of weights and o to bf16, 2^-12 for the fp32 sums); and the mean error, where the bf16 roundings of some 10^5
elements cancel to under 2^-15, is held to 2^-12 of the mean, the share of the sums alone."""
import math

import pytest
import torch

import paper_2609_30884_gb300 as crf
from tests.test_gpu_extend import BF16, DEV, PAGE, Setup, gen, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


def repeated(ctx, hkv, dim, rows, pages, times, chunks):
    """(error of o, its tolerance, o in 64 bits, error of lse, its tolerance) of `chunks` equal requests of `rows` rows
    over `pages` pages `times` times."""
    g = gen(81)
    k = normal(g, pages, hkv, PAGE, dim)
    v = (normal(g, pages, hkv, PAGE, dim, dtype=torch.float32) * 0.5 + 1).to(BF16)  # of one sign mostly
    q = normal(g, rows * chunks, hkv, dim)
    table = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
    b = crf.Chunks([table.repeat(times)] * chunks, [rows] * chunks, [0] * chunks, [pages * PAGE * times] * chunks)
    pool, out, lse = crf.KVPool([k], [v]), torch.empty_like(q), torch.empty(rows * chunks, hkv, device=DEV)
    ctx.chunk_attention(pool, 0, b, q, out, ctx.chunk_attention_workspace(pool, b, hkv, causal=False), lse=lse, causal=False)
    ctx.check()
    kk, vv = (x.transpose(0, 1).reshape(hkv, -1, dim).double() for x in (k, v))
    z = torch.einsum("rhd,hnd->rhn", q.double(), kk) * dim**-0.5
    w = z.softmax(-1)
    want, size = torch.einsum("rhn,hnd->rhd", w, vv), torch.einsum("rhn,hnd->rhd", w, vv.abs())
    reach = torch.einsum("rhd,hnd->rhn", q.double().abs(), kk.abs()).amax(-1) * dim**-0.5
    lse64 = z.logsumexp(-1) + math.log(times)
    return (out.double() - want, size * (2.0**-8 + 2.0**-12) + want.abs() * 2.0**-8 * 1.01, want,
            lse.double() - lse64, 2.0**-16 * reach + 2.0**-17 * (1 + lse64.abs()))


# (kv heads, head size, rows, requests): 152 tiles of 256 rows, a request's all; single tokens
@pytest.mark.parametrize("hkv,dim,rows,chunks", [(4, 128, 9728, 1), (4, 64, 9728, 1), (2, 128, 1, 64)])
@pytest.mark.parametrize("times", [256, 4096])
def test_sums_over_many_tiles(ctx, hkv, dim, rows, chunks, times):
    err, tol, want, lse_err, lse_tol = repeated(ctx, hkv, dim, rows, 64, times, chunks)  # 2^18 and 2^22 keys
    assert bool((err.abs() <= tol).all()), float((err.abs() - tol).max())
    assert abs(float(err.sum() / want.sum())) <= 2.0**-12
    assert bool((lse_err.abs() <= lse_tol).all()), float((lse_err.abs() - lse_tol).max())


# 19 query tiles of 8 heads for 152 SMs: sums start anew twice within a tile's keys, which the rows see in part
@pytest.mark.parametrize("dim,rows,pos,window", [(64, 4864, 35136, 0), (128, 4864, 35136, 0), (64, 4864, 35136, 25000),
                                                 (128, 4864, 60000, 33333), (64, 4864, 12000, 0)])
def test_long_tiles_of_seen_and_unseen_keys(ctx, dim, rows, pos, window):
    s = Setup(82, 8, 8, dim, [(rows, pos)], window=window)
    out, lse = s.run(ctx)
    s.verify(out, lse)
    again, lse2 = s.run(ctx)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    ctx.check()


@pytest.mark.parametrize("up", [1, -1])
def test_long_rising_and_falling_scores(ctx, up):
    """The maximum of later sums leaves the totals of earlier ones far behind, or never changes."""
    s = Setup(83, 8, 8, 64, [(4864, 35136)], poison=False)
    n, t = 40000, s.tables[0].long()
    j = torch.arange(n, device=DEV)
    s.k[t[j // PAGE], :, j % PAGE] = (s.k[t[j // PAGE], :, j % PAGE].float() * 0.1 + (up * j / 2000.0)[:, None, None]).to(BF16)
    s.q.copy_((s.q.float().abs() * 0.5).to(BF16))
    s.verify(*s.run(ctx))
    ctx.check()


def test_infinite_values_in_long_tiles(ctx):
    """An infinity or NaN of v before, between and behind the starts of a sum reaches the rows that see it and no other."""
    s = Setup(84, 8, 8, 64, [(4864, 35136)], poison=False)
    out, lse = s.run(ctx)
    t, hit = s.tables[0].long(), torch.zeros_like(out, dtype=torch.bool)
    for at, head, col, e in ((5, 0, 3, math.inf), (20000, 2, 7, -math.inf), (30001, 3, 9, math.nan), (36000, 4, 0, math.inf),
                             (39999, 7, 63, math.nan)):
        s.v[t[at // PAGE], head, at % PAGE, col] = e
        hit[max(0, at - 35136):, head, col] = True
    got, lse2 = s.run(ctx)
    assert not bool(got[hit].isfinite().any()) and torch.equal(torch.where(hit, 0, out), torch.where(hit, 0, got))
    assert torch.equal(lse, lse2)
    ctx.check()
