"""The time of a call over a shared prefix does not depend on what lies in cache slots that hold no key. The bound is a factor of two, far
from what timing noise does and from what it was where such slots were taken for values to give back (over ten)."""
import math

import pytest
import torch

import paper_2609_30884_gb300 as crf
from tests.test_gpu_extend import PAGE
from tests.test_gpu_extend_wider import Shared, shared_kernel

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


def time_of(ctx, s, out):
    b, p = s.batch(), s.prefixes()
    ws = ctx.prefix_attention_workspace(s.pool, b, p, s.hq)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    times = []
    for _ in range(12):
        torch.cuda._sleep(200000)
        start.record()
        for _ in range(5):
            ctx.prefix_attention(s.pool, 0, b, p, s.q, out, ws)
        end.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(end))
    return sorted(times[2:])[5]


@pytest.mark.parametrize("hq,hkv,dim,groups", [(28, 4, 128, [(15000, [(1, 19 * i + 5, 0) for i in range(32)])]), (12, 2, 64, [(9003, [(3, 7, 0)] * 30)])])
def test_time_over_slots_without_keys(ctx, hq, hkv, dim, groups):
    s = Shared(51, hq, hkv, dim, groups, poison=False)
    assert shared_kernel(ctx, lambda: s.run(ctx))
    want = torch.empty_like(s.q)
    finite = time_of(ctx, s, want)
    for (_, _, n), t in zip(s.chunks, s.tables):
        if n % PAGE:
            last = t[n // PAGE].long()
            s.k[last, :, n % PAGE:], s.v[last, :, n % PAGE:] = math.nan, math.nan
    got = torch.empty_like(s.q)
    unwritten = time_of(ctx, s, got)
    ctx.check()
    assert torch.equal(got, want)
    assert unwritten < 2 * finite, (unwritten, finite)
