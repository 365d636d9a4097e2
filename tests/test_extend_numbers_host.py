"""Numbers that the binding passes on in 32 bits: one that does not fit is refused, and is never another one to the library."""
import ctypes

import pytest
import torch

import paper_2609_30884_gb300 as crf

WRAPS = [1 << 31, (1 << 32) + 5, (1 << 40) + 16, -(1 << 31) - 1, -(1 << 32) + 5]
TABLE = torch.arange(8, dtype=torch.int32)


@pytest.mark.parametrize("big", WRAPS)
def test_descriptors_refuse_numbers_beyond_32_bits(big):
    for bad in (lambda: crf.Chunks([TABLE], [big], [0], [60]), lambda: crf.Chunks([TABLE], [1], [big], [60]),
                lambda: crf.Chunks([TABLE], [1], [5], [big]), lambda: crf.Chunks([TABLE], [0], [big]),
                lambda: crf.Chunks([TABLE], [1], [(1 << 31) - 1]), lambda: crf.PageTables([TABLE], [big]),
                lambda: crf.Rope(big), lambda: crf.Rope(64, rot_dim=big)):
        with pytest.raises(ValueError):
            bad()


def test_descriptors_pass_on_what_fits():
    # the library refuses the negative ones by itself
    c = crf.Chunks([TABLE], [1], [-3], [-(1 << 31)])
    assert (c.c[0].n_new, c.c[0].pos, c.c[0].n_keys) == (1, -3, -(1 << 31))
    assert crf.Chunks([TABLE], [1], [(1 << 31) - 2]).c[0].n_keys == (1 << 31) - 1
    assert crf.PageTables([TABLE], [-1]).c[0].n_tokens == -1


@pytest.mark.parametrize("big", WRAPS)
def test_calls_refuse_numbers_beyond_32_bits(big):
    class NoCall:
        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")

    ctx = crf.Context.__new__(crf.Context)
    ctx.device, ctx.h, ctx.lib, ctx._parts = -1, None, NoCall(), ctypes.create_string_buffer(3 * crf._HEADS)
    pages = torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16)
    pool, b, x = crf.KVPool([pages], [pages]), crf.Chunks([TABLE], [3], [0]), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(256, dtype=torch.uint8)
    for bad in (lambda: ctx.chunk_attention(pool, 0, b, x, torch.zeros_like(x), ws, window=big, stream=0),
                lambda: ctx.chunk_attention_workspace(pool, b, 2, window=big), lambda: ctx.chunk_attention_workspace(pool, b, big),
                lambda: ctx.pages_workspace(big, crf.PageTables([TABLE], [9]))):
        with pytest.raises(ValueError):
            bad()
