"""The alternatives' two outputs, as the binding takes them: of one shape, whatever their number of elements (tensors of the host; the library is a
stand-in that notes what it is called with)."""
import ctypes

import pytest
import torch

import paper_2609_30884_gb300 as crf


class Noted:
    def __init__(self):
        self.calls = []

    def crf_logprobs(self, *a):
        self.calls.append(a)
        return 0


@pytest.fixture
def ctx():
    c = crf.Context.__new__(crf.Context)
    c.lib, c.h, c.device = Noted(), None, -1  # the host's tensors are on device -1
    yield c
    c.h = ctypes.c_void_p()


Z = torch.zeros(3, 50)


@pytest.mark.parametrize("shape", [(4, 3), (12,), (1, 12), (2, 6), (3, 5), (3, 4, 1), (3, 2, 2), ()])
def test_alternatives_of_two_shapes_are_refused(ctx, shape):
    ids, tops = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(shape)
    with pytest.raises(ValueError):
        ctx.logprobs(Z, top_ids=ids, top_logprobs=tops, stream=0)
    with pytest.raises(ValueError):
        ctx.logprobs(Z, top_ids=tops.int(), top_logprobs=ids.float(), stream=0)
    assert not ctx.lib.calls


def test_alternatives_that_are_taken(ctx):
    ids, tops = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 4)
    for kw in (dict(top_ids=ids, top_logprobs=tops), dict(top_ids=ids), dict(top_logprobs=tops)):
        ctx.logprobs(Z, stream=0, **kw)
        call = ctx.lib.calls.pop()
        assert call[10] == 4 and call[11] == (ids.data_ptr() if "top_ids" in kw else None)
        assert call[12] == (tops.data_ptr() if "top_logprobs" in kw else None)
    ctx.logprobs(Z, stream=0, lse=torch.zeros(3))
    assert ctx.lib.calls.pop()[10] == 0
