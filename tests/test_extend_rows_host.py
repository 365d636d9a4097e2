"""Rows beyond 32 bits: the calls on rows of heads refuse them, and do not pass on what is left of their number (tensors without memory)."""
import ctypes

import pytest
import torch

import paper_2609_30884_gb300 as crf


class NoCall:
    def __getattr__(self, name):
        return lambda *a: pytest.fail(f"{name} was called")


@pytest.mark.parametrize("rows", [1 << 31, (1 << 32) + 5, (1 << 33)])
def test_rows_beyond_32_bits_are_refused(rows):
    ctx = crf.Context.__new__(crf.Context)
    ctx.lib, ctx.h, ctx.device = NoCall(), None, -1  # such tensors are on device -1
    ctx._parts, ctx._norms, ctx._dgains = ctypes.create_string_buffer(4 * crf._HEADS), ctypes.create_string_buffer(2 * crf._NORM), (ctypes.c_void_p * 2)()
    x = torch.empty(rows, 1, 2, dtype=torch.bfloat16, device="meta")
    w, pos = torch.empty(2, dtype=torch.bfloat16, device="meta"), torch.empty(rows, dtype=torch.int32, device="meta")
    dgain, ws, rope = torch.empty(2, device="meta"), torch.empty(1 << 20, dtype=torch.uint8, device="meta"), crf.Rope(2)
    for call in (lambda: ctx.rotary(rope, pos, x, stream=0), lambda: ctx.rotary(rope, pos, x, k=x, stream=0), lambda: ctx.norm_rotary(rope, pos, x, w, stream=0),
                 lambda: ctx.norm_rotary_grad(rope, pos, x, w, x, x, dgain, ws, stream=0), lambda: ctx.norm_rotary_workspace(rope, rows)):
        with pytest.raises(ValueError):
            call()
    ctx.h = ctypes.c_void_p()
