"""Attention's scale at the ends of fp32: what the kernel could only turn into infinities, or the binding into the default,
is refused."""
import ctypes

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300 import abi
from tests.test_extend_host import A16, call_attention, ctx, lib  # noqa: F401

LOG2E = 1.4426950408889634


@pytest.mark.parametrize("scale", [3.4e38, 2.4e38])
def test_a_scale_whose_log2_form_is_infinite_is_refused(lib, ctx, scale):  # noqa: F811
    assert ctypes.c_float(scale).value < float("inf") and ctypes.c_float(scale * LOG2E).value == float("inf")
    assert call_attention(lib, ctx, scale=scale) == abi.EINVAL
    assert b"scale" in lib.crf_last_error()


@pytest.mark.parametrize("scale", [2.3e38, 1.0, 1e-38, 2.0**-149])
def test_scales_in_range_get_past_that_check(lib, ctx, scale):  # noqa: F811
    # what stands behind it is refused instead: a misaligned workspace
    assert call_attention(lib, ctx, scale=scale, ch=((1, 100000, 100001, A16),), ws=A16 + 16) == abi.EINVAL
    assert b"workspace" in lib.crf_last_error()


@pytest.mark.parametrize("scale", [1e-46, 2.0**-150, 5e-324])
def test_a_scale_that_float32_has_not_is_not_taken_for_the_default(scale):
    class NoCall:
        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")

    c = crf.Context.__new__(crf.Context)
    c.device, c.h, c.lib, c._parts = -1, None, NoCall(), ctypes.create_string_buffer(3 * crf._HEADS)
    pages, x = torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="scale"):
        c.chunk_attention(crf.KVPool([pages], [pages]), 0, crf.Chunks([torch.arange(8, dtype=torch.int32)], [3], [0]), x,
                          torch.zeros_like(x), torch.zeros(256, dtype=torch.uint8), scale=scale, stream=0)
