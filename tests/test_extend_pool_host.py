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


def wrong_pools():
    k, v = (lambda: pages(5, 2, 16, 64)), (lambda: pages(5, 2, 16, 64))  # noqa: E731
    return {
        "V of fewer pages": ([k(), k()], [v(), pages(4, 2, 16, 64)]),
        "K of fewer pages in a later layer": ([k(), pages(4, 2, 16, 64)], [v(), v()]),
        "V of fewer heads": ([k()], [pages(5, 1, 16, 64)]),
        "another layer's head size": ([k(), pages(5, 2, 16, 32)], [v(), v()]),
        "a flat later layer": ([k(), k().view(5, 2048)], [v(), v()]),
        "V flat": ([k()], [v().view(-1)]),
        "pages of eight": ([pages(5, 2, 8, 64)], [pages(5, 2, 8, 64)]),
        "fp16": ([pages(5, 2, 16, 64, dtype=torch.float16)], [pages(5, 2, 16, 64, dtype=torch.float16)]),
        "V of fp32": ([k()], [pages(5, 2, 16, 64, dtype=torch.float32)]),
        "every other page": ([pages(10, 2, 16, 64)[::2]], [v()]),
        "V of heads outside": ([k()], [pages(2, 5, 16, 64).transpose(0, 1)]),
        "V elsewhere": ([k()], [torch.empty(5, 2, 16, 64, dtype=BF16, device="meta")]),
    }


@pytest.mark.parametrize("name", sorted(wrong_pools()))
def test_a_pool_that_is_not_pages_throughout_is_refused(ctx, name):
    """Its tensors' addresses would be read and written by layer 0's keys' shape, behind the end of a smaller one."""
    pool = crf.KVPool(*wrong_pools()[name])
    for call in extension_calls(ctx, pool).values():
        with pytest.raises(ValueError):
            call()


def test_layers_of_more_pages_than_the_first_are_fine(ctx):
    pool = crf.KVPool([pages(5, 2, 16, 64), pages(7, 2, 16, 64)], [pages(6, 2, 16, 64), pages(5, 2, 16, 64)])
    with pytest.raises(AssertionError, match="was called"):
        extension_calls(ctx, pool)["append"]()


@pytest.mark.parametrize("layers", [(2, 1)])
def test_layers_without_values_are_refused(ctx, layers):
    pool = crf.KVPool([pages(5, 2, 16, 64) for _ in range(layers[0])], [pages(5, 2, 16, 64) for _ in range(layers[1])])
    for call in extension_calls(ctx, pool).values():
        with pytest.raises(ValueError):
            call()
