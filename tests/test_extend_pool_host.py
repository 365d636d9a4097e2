"""What the binding asks of a page pool before its addresses go to the calls that extend a cache (no GPU)."""
import ctypes

import pytest
import torch

import paper_2609_30884_gb300 as crf

BF16 = torch.bfloat16


class NoCall:
    """In place of the library: a call that gets this far was not refused."""

    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


@pytest.fixture()
def ctx():
    c = crf.Context.__new__(crf.Context)
    c.device, c.h, c.lib = -1, None, NoCall()  # tensors in host memory are on "device" -1
    c._parts = ctypes.create_string_buffer(3 * crf._HEADS)
    return c


def pages(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


def extension_calls(ctx, pool, layer=0, heads=2, dim=64):
    """Every call that reads or writes the pool, with arguments that fit [.., 2, 16, 64]."""
    t, x = torch.zeros(4, dtype=torch.int32), torch.zeros(3, heads, dim, dtype=BF16)
    ws, b = torch.zeros(256, dtype=torch.uint8), crf.Chunks([t], [3], [0])
    tables, refs = crf.PageTables([t], [16], [t.clone()]), torch.zeros(pool.num_pages, dtype=torch.int32)
    return {
        "append": lambda: ctx.cache_append(pool, layer, b, x, x, stream=0),
        "attention": lambda: ctx.chunk_attention(pool, layer, b, x, torch.zeros_like(x), ws, stream=0),
        "workspace": lambda: ctx.chunk_attention_workspace(pool, b, heads),
        "fork": lambda: ctx.pages_fork(pool, refs, tables, ws, stream=0),
        "compact": lambda: ctx.pages_compact(pool, refs, tables, ws, stream=0),
    }


CALLS = ("append", "attention", "workspace", "fork", "compact")


@pytest.mark.parametrize("call", CALLS)
def test_a_pool_of_pages_reaches_the_library(ctx, call):
    pool = crf.KVPool([pages(5, 2, 16, 64)] * 2, [pages(5, 2, 16, 64)] * 2)
    with pytest.raises(AssertionError, match="was called"):
        extension_calls(ctx, pool, layer=1)[call]()


@pytest.mark.parametrize("shape", [(5, 2 * 16 * 64), (5, 2, 16 * 64), (5, 2 * 16, 64), (5 * 2 * 16 * 64,), (5, 1, 2, 16, 64)])
def test_flat_views_of_the_pages_make_a_pool(ctx, shape):
    k, v = pages(5, 2, 16, 64), pages(5, 2, 16, 64)
    pool = crf.KVPool([k.view(shape)], [v.view(shape)])
    assert pool.num_pages == shape[0] and pool.c.num_pages == shape[0]
    assert (pool.c.k_pages[0], pool.c.v_pages[0]) == (k.data_ptr(), v.data_ptr())
    for name, call in extension_calls(ctx, pool).items():
        with pytest.raises(ValueError, match="kv heads, 16, head_dim"):
            call()
