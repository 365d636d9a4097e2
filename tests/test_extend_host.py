"""Calls that extend a recovered cache, as far as they go without a GPU: struct layouts, every refusal of
the C ABI (made before the context's device is touched, so a zeroed stand-in serves as the context) and the
binding's own checks."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300 import abi, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "crf.h")
EINVAL, ESHAPE, EUNSUPPORTED, ENOMEM = abi.EINVAL, abi.ESHAPE, abi.EUNSUPPORTED, abi.ENOMEM

STRUCTS = {
    "crf_rope": (abi.Rope, ["head_dim", "rot_dim", "layout", "scaling", "theta", "factor", "low", "high", "original",
                            "magnitude"]),
    "crf_heads": (abi.Heads, ["x", "out", "heads", "x_row", "x_head", "out_row", "out_head"]),
    "crf_chunk": (abi.Chunk, ["n_new", "pos", "n_keys", "page_table"]),
    "crf_pages": (abi.Pages, ["n_tokens", "table", "out"]),
}


def test_struct_layouts_match_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{HEADER}"', "int main(void){"]
    for name, (_, fields) in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f in fields]
    lines.append('printf("enums %d %d %d %d %d %d %d\\n", CRF_MAX_CHUNKS, CRF_MAX_TABLES, CRF_BF16, CRF_FP16, CRF_FP32, '
                 "CRF_ROPE_INTERLEAVED, CRF_ROPE_BANDS);")
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run([cc, str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.splitlines()
    got = dict(l.split(" ", 1) for l in out)
    for name, (cls, fields) in STRUCTS.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f in fields:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, f"{name}.{f}"
    assert got["enums"] == (f"{abi.MAX_CHUNKS} {abi.MAX_TABLES} {abi.BF16} {abi.FP16} {abi.FP32} "
                            f"{abi.ROPE_LAYOUTS['interleaved']} {abi.ROPE_SCALINGS['bands']}")


@pytest.fixture(scope="module")
def lib():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        if not os.path.exists(abi.LIB_PATH):
            pytest.skip("no nvcc and no prebuilt library")
    else:
        build.build()
    return abi.load()


@pytest.fixture()
def ctx():
    # device 0, 152 SMs, everything else zero: refusals read no more of a context
    buf = ctypes.create_string_buffer(4096)
    ctypes.memmove(buf, (ctypes.c_int * 2)(0, 152), 8)
    return buf


def ref(s):
    return ctypes.byref(s)


def rope(**kw):
    return crf.Rope(**{**dict(head_dim=64), **kw}).c


A16 = 1 << 20  # an aligned address that nothing reads


def heads(**kw):
    d = dict(x=A16, out=A16 + 4096, heads=4, x_row=256, x_head=64, out_row=256, out_head=64)
    d.update(kw)
    return abi.Heads(*(d[f] for f in ("x", "out", "heads", "x_row", "x_head", "out_row", "out_head")))


def pool(num_pages=9, k=A16, v=A16):
    c = abi.KVPool()
    c._k, c._v = (ctypes.c_void_p * 1)(k), (ctypes.c_void_p * 1)(v)
    c.k_pages, c.v_pages, c.num_pages = c._k, c._v, num_pages
    return c


def chunks(*c):
    arr = (abi.Chunk * max(1, len(c)))()
    for i, x in enumerate(c):
        arr[i] = abi.Chunk(*x)
    return arr


def call_rotary(lib, ctx, r=None, p=None, n_parts=1, type=abi.BF16, rows=3, positions=A16):
    parts = (abi.Heads * 2)(*(p or (heads(), heads())))
    return lib.crf_rotary(ctx, ref(r or rope()), parts, n_parts, type, rows, positions, 0, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rot_dim=63), EUNSUPPORTED), (dict(rot_dim=0), EUNSUPPORTED), (dict(rot_dim=66), EUNSUPPORTED),
    (dict(head_dim=258, rot_dim=2), EUNSUPPORTED), (dict(head_dim=1, rot_dim=2), EUNSUPPORTED),
    (dict(theta=0.0), EINVAL), (dict(theta=-1.0), EINVAL), (dict(theta=math.inf), EINVAL), (dict(theta=math.nan), EINVAL),
    (dict(magnitude=math.nan), EINVAL), (dict(magnitude=1e300), EINVAL),
    (dict(scaling="linear", factor=0.5), EINVAL), (dict(scaling="linear", factor=math.nan), EINVAL),
    (dict(scaling="linear", factor=math.inf), EINVAL), (dict(scaling="base", rot_dim=2, factor=2.0), EUNSUPPORTED),
    (dict(scaling="bands", factor=2.0, low=4.0, high=4.0), EINVAL), (dict(scaling="bands", factor=2.0, low=-1.0), EINVAL),
    (dict(scaling="bands", factor=2.0, high=math.inf), EINVAL), (dict(scaling="bands", factor=2.0, original=0.0), EINVAL),
])
def test_rope_refusals(lib, ctx, kw, status):
    assert call_rotary(lib, ctx, rope(**kw)) == status


@pytest.mark.parametrize("kw", [
    dict(theta=5e-324), dict(theta=1e-308, rot_dim=64), dict(theta=1e300, scaling="base", factor=1e20, rot_dim=4),
    dict(scaling="base", factor=1e308, rot_dim=4),
])
def test_rope_refuses_a_base_out_of_range(lib, ctx, kw):
    # the frequencies or the base itself would be infinite
    assert call_rotary(lib, ctx, rope(**kw)) == EINVAL


def test_rope_unknown_layout_or_scaling(lib, ctx):
    for field in ("layout", "scaling"):
        for bad in (-1, 4):
            r = rope()
            setattr(r, field, bad)
            assert call_rotary(lib, ctx, r) == EINVAL
    with pytest.raises(ValueError):
        crf.Rope(64, layout="pairs")
    with pytest.raises(ValueError):
        crf.Rope(64, scaling="other")


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(heads=0), EINVAL), (dict(heads=65536), EINVAL),
    (dict(x_row=-1), EINVAL), (dict(out_head=-64), EINVAL), (dict(x=A16 + 1), EINVAL), (dict(x_row=1 << 41), EINVAL),
    (dict(out_row=0), ESHAPE), (dict(out_head=32), ESHAPE), (dict(out_row=255), ESHAPE),
    (dict(x=A16, out=A16, x_row=512), ESHAPE),
])
def test_rotary_refusals(lib, ctx, kw, status):
    assert call_rotary(lib, ctx, p=(heads(**kw), heads())) == status
    assert call_rotary(lib, ctx, p=(heads(), heads(**kw)), n_parts=2) == status


def test_rotary_refuses_rows_too_far_apart_to_multiply(lib, ctx):
    # (rows - 1) x row is over 2^63: rows and heads interleave, whatever the product wraps to
    far = heads(out_row=1 << 40, out_head=1 << 40)
    for rows in ((1 << 23) + 1, (1 << 24) + 1, (1 << 31) - 1):
        assert call_rotary(lib, ctx, p=(far, heads()), rows=rows) == ESHAPE


def test_rotary_argument_refusals(lib, ctx):
    assert lib.crf_rotary(None, ref(rope()), ref(heads()), 1, 0, 1, A16, 0, None) == EINVAL
    assert lib.crf_rotary(ctx, None, ref(heads()), 1, 0, 1, A16, 0, None) == EINVAL
    assert lib.crf_rotary(ctx, ref(rope()), None, 1, 0, 1, A16, 0, None) == EINVAL
    assert call_rotary(lib, ctx, n_parts=0) == EINVAL and call_rotary(lib, ctx, n_parts=3) == EINVAL
    assert call_rotary(lib, ctx, type=3) == EUNSUPPORTED and call_rotary(lib, ctx, type=-1) == EUNSUPPORTED
    assert call_rotary(lib, ctx, positions=A16 + 1) == EINVAL
    assert call_rotary(lib, ctx, rows=-1) == EINVAL and call_rotary(lib, ctx, positions=None) == EINVAL
    assert call_rotary(lib, ctx, rows=0, positions=None) == abi.OK  # nothing to do


def call_append(lib, ctx, r=True, pl=None, layer=0, hkv=2, d=64, ch=((3, 5, 8, A16),), q=None, k=None, v=None, n=None):
    c = chunks(*ch)
    return lib.crf_cache_append(ctx, ref(rope()) if r is True else r, ref(pl or pool()), layer, hkv, d, c,
                                len(ch) if n is None else n, q, ref(k or heads(heads=2)), ref(v or heads(heads=2)), None)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), EINVAL), (dict(d=96), EUNSUPPORTED), (dict(hkv=0), EINVAL), (dict(pl=pool(0)), EINVAL),
    (dict(pl=pool(1 << 30), hkv=2), EUNSUPPORTED), (dict(pl=pool(k=None)), EINVAL), (dict(pl=pool(v=A16 + 8)), EINVAL),
    (dict(n=0), EINVAL), (dict(n=129), EINVAL), (dict(ch=((-1, 0, 0, A16),)), EINVAL), (dict(ch=((1, -1, 0, A16),)), EINVAL),
    (dict(ch=((1, 1 << 30, 1, A16),)), EINVAL), (dict(ch=((1, 0, 1, None),)), EINVAL),
    (dict(ch=((1 << 30, 0, 0, A16), (1, 0, 1, A16))), EINVAL),
    (dict(k=heads(heads=3)), ESHAPE), (dict(v=heads(heads=4)), ESHAPE), (dict(k=heads(heads=2, x=None)), EINVAL),
    (dict(d=128), ESHAPE), (dict(r=None, q=ref(heads())), EINVAL), (dict(q=ref(heads(out=None))), EINVAL),
    (dict(q=ref(heads(out_row=8))), ESHAPE),
])
def test_append_refusals(lib, ctx, kw, status):
    assert call_append(lib, ctx, **kw) == status


def test_append_of_no_rows_is_nothing(lib, ctx):
    assert call_append(lib, ctx, ch=((0, 0, 0, None), (0, 7, 7, None))) == abi.OK


def call_attention(lib, ctx, pl=None, layer=0, hkv=2, d=64, ch=((3, 5, 8, A16),), q=None, scale=0.0, window=0, ws=A16,
                   ws_bytes=1 << 30, n=None, lse=None):
    c = chunks(*ch)
    return lib.crf_chunk_attention(ctx, ref(pl or pool()), layer, hkv, d, c, len(ch) if n is None else n, ref(q or heads()),
                                   lse, scale, 1, window, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), EINVAL), (dict(d=80), EUNSUPPORTED), (dict(hkv=3), ESHAPE), (dict(hkv=0), EINVAL), (dict(window=-1), EINVAL),
    (dict(scale=-1.0), EINVAL), (dict(scale=math.nan), EINVAL), (dict(scale=math.inf), EINVAL), (dict(n=0), EINVAL), (dict(n=129), EINVAL),
    (dict(ch=((1, 5, -1, A16),)), EINVAL), (dict(ch=((1, 5, (1 << 30) + 1, A16),)), EINVAL), (dict(ch=((1, 5, 6, None),)), EINVAL),
    (dict(q=heads(x=A16 + 2)), EINVAL), (dict(q=heads(x_row=260)), EUNSUPPORTED), (dict(q=heads(out_head=68)), EUNSUPPORTED),
    (dict(q=heads(out=A16)), EINVAL), (dict(q=heads(out_row=64)), ESHAPE), (dict(q=heads(heads=3)), ESHAPE),
    (dict(pl=pool(k=None)), EINVAL), (dict(ch=((1, 5, 6, A16 + 2),)), EINVAL), (dict(lse=A16 + 2), EINVAL),
    (dict(ch=((1, 1 << 26, (1 << 26) + 1, A16),)), EUNSUPPORTED),
    (dict(ch=((1 << 29, 0, 1 << 20, A16),)), EUNSUPPORTED),
])
def test_attention_refusals(lib, ctx, kw, status):
    assert call_attention(lib, ctx, **kw) == status


def test_strides_of_axes_of_one_are_not_refused(lib, ctx):
    # what stands behind the strides is refused instead: a missing workspace, misaligned positions
    long = dict(ch=((1, 100000, 100001, A16),), ws=A16 + 16)
    assert call_attention(lib, ctx, q=heads(x_row=3, out_row=0), **long) == EINVAL
    assert b"workspace" in lib.crf_last_error()
    one = heads(heads=1, x_head=5, out_head=0)
    assert call_attention(lib, ctx, hkv=1, q=one, **long) == EINVAL
    assert b"workspace" in lib.crf_last_error()
    bad = heads(out=None)
    assert call_rotary(lib, ctx, p=(heads(x_row=-1, out_row=0), bad), n_parts=2, rows=1) == EINVAL
    assert b"part 1" in lib.crf_last_error()
    assert call_rotary(lib, ctx, p=(heads(heads=1, x_head=-1, out_head=0), bad), n_parts=2) == EINVAL
    assert b"part 1" in lib.crf_last_error()


def test_attention_workspace(lib, ctx):
    n = ctypes.c_size_t()
    long = chunks((1, 100000, 100001, A16))
    assert lib.crf_chunk_attention_workspace_size(ctx, 4, 2, 64, long, 1, 1, 0, ref(n)) == abi.OK
    need = n.value
    if need:
        assert call_attention(lib, ctx, ch=((1, 100000, 100001, A16),), ws_bytes=need - 1) == ENOMEM
        assert call_attention(lib, ctx, ch=((1, 100000, 100001, A16),), ws=None) == EINVAL
        assert call_attention(lib, ctx, ch=((1, 100000, 100001, A16),), ws=A16 + 16) == EINVAL
    assert lib.crf_chunk_attention_workspace_size(ctx, 4, 2, 64, long, 1, 1, 0, None) == EINVAL
    assert lib.crf_chunk_attention_workspace_size(ctx, 5, 2, 64, long, 1, 1, 0, ref(n)) == ESHAPE


def test_attention_of_no_rows_is_nothing(lib, ctx):
    assert call_attention(lib, ctx, ch=((0, 0, 0, None), (0, 9, 9, None)), ws=None, ws_bytes=0) == abi.OK


def tables(*t):
    arr = (abi.Pages * max(1, len(t)))()
    for i, x in enumerate(t):
        arr[i] = abi.Pages(*x)
    return arr


PAGE_BAD = [
    (dict(t=((-1, A16, A16),)), EINVAL), (dict(t=(((1 << 30) + 1, A16, A16),)), EINVAL), (dict(t=((1, None, A16),)), EINVAL),
    (dict(t=((1, A16 + 1, A16),)), EINVAL), (dict(refs=A16 + 2), EINVAL),
    (dict(n=0), EINVAL), (dict(n=513), EINVAL), (dict(refs=None), EINVAL), (dict(refs_out=None), EINVAL),
    (dict(ws=None), EINVAL), (dict(ws=A16 + 64), EINVAL), (dict(ws_bytes=64), ENOMEM),
]
POOL_BAD = [
    (dict(t=((1, A16, None),)), EINVAL), (dict(layers=0), EINVAL), (dict(hkv=0), EINVAL), (dict(d=32), EUNSUPPORTED),
    (dict(pl=pool(0)), EINVAL), (dict(pl=pool(v=None)), EINVAL),
]


def call_pages(lib, ctx, op, pl=None, layers=1, hkv=2, d=64, refs=A16, refs_out=A16, t=((40, A16, A16),), n=None, ws=A16,
               ws_bytes=1 << 30):
    arr, n = tables(*t), len(t) if n is None else n
    if op == "release":
        return lib.crf_pages_release(ctx, 9, refs, refs_out, arr, n, ws, ws_bytes, None)
    pl = pl or pool()
    if op == "fork":
        return lib.crf_pages_fork(ctx, ref(pl), layers, hkv, d, refs, refs_out, arr, n, 0, ws, ws_bytes, None)
    return lib.crf_pages_compact(ctx, ref(pl), layers, hkv, d, refs, refs_out, arr, n, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", PAGE_BAD)
@pytest.mark.parametrize("op", ["fork", "compact", "release"])
def test_page_refusals(lib, ctx, op, kw, status):
    assert call_pages(lib, ctx, op, **kw) == status


@pytest.mark.parametrize("kw,status", POOL_BAD)
@pytest.mark.parametrize("op", ["fork", "compact"])
def test_page_pool_refusals(lib, ctx, op, kw, status):
    assert call_pages(lib, ctx, op, **kw) == status


def test_page_workspace_size(lib, ctx):
    n = ctypes.c_size_t()
    assert lib.crf_pages_workspace_size(ctx, 1000, tables((40, A16, A16)), 1, ref(n)) == abi.OK and n.value >= 4 * 1000
    assert n.value % 256 == 0
    assert lib.crf_pages_workspace_size(ctx, 0, tables((40, A16, A16)), 1, ref(n)) == EINVAL
    assert lib.crf_pages_workspace_size(ctx, 10, tables((-1, A16, A16)), 1, ref(n)) == EINVAL


# ---------------------------------------------------------------------------------------------- the binding
def test_chunks_marshalling():
    pts = [torch.arange(4, dtype=torch.int32), torch.arange(2, dtype=torch.int32)]
    c = crf.Chunks(pts, [3, 1], [40, 9])
    assert (c.n, c.rows) == (2, 4)
    assert [(c.c[i].n_new, c.c[i].pos, c.c[i].n_keys) for i in range(2)] == [(3, 40, 43), (1, 9, 10)]
    assert [c.c[i].page_table for i in range(2)] == [t.data_ptr() for t in pts]
    assert c.append_ok and c.attend_ok
    assert not crf.Chunks(pts, [3, 1], [62, 9]).append_ok          # 65 positions need a fifth page
    assert not crf.Chunks(pts, [3, 1], [40, 9], [43, 33]).attend_ok
    assert crf.Chunks(pts, [0, 1], [999, 9], [999, 10]).append_ok  # no row, nothing read
    with pytest.raises(ValueError):
        crf.Chunks(pts, [1], [0, 0])
    with pytest.raises(ValueError):
        crf.Chunks([pts[0].long()], [1], [0])
    with pytest.raises(ValueError):
        crf.Chunks([torch.arange(8, dtype=torch.int32)[::2]], [1], [0])


def test_page_tables_marshalling():
    t, o = torch.arange(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    p = crf.PageTables([t], [40], [o])
    assert (p.c[0].n_tokens, p.c[0].table, p.c[0].out) == (40, t.data_ptr(), o.data_ptr())
    assert crf.PageTables([t], [48]).c[0].out is None
    for bad in (lambda: crf.PageTables([t], [49]), lambda: crf.PageTables([t], [40], [o[:2]]),
                lambda: crf.PageTables([t, t], [40]), lambda: crf.PageTables([t.float()], [40])):
        with pytest.raises(ValueError):
            bad()


def test_a_context_of_a_gpu_refuses_tensors_elsewhere(lib):
    """The binding looks at where tensors are before it takes their addresses."""
    ctx = crf.Context.__new__(crf.Context)
    ctx.device, ctx.h, ctx.lib = 0, None, lib
    ctx._parts = ctypes.create_string_buffer(3 * crf._HEADS)
    t, x = torch.zeros(4, dtype=torch.int32), torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    ws = torch.zeros(256, dtype=torch.uint8)
    pool = crf.KVPool([torch.zeros(4, 3, 16, 64, dtype=torch.bfloat16)], [torch.zeros(4, 3, 16, 64, dtype=torch.bfloat16)])
    assert (pool.n_kv_heads, pool.head_dim) == (3, 64)
    with pytest.raises(ValueError):
        ctx.rotary(crf.Rope(64), t, x)
    with pytest.raises(ValueError):
        ctx.cache_append(pool, 0, crf.Chunks([t], [2], [0]), x, x)
    with pytest.raises(ValueError):
        ctx.chunk_attention(pool, 0, crf.Chunks([t], [2], [0]), x, torch.zeros_like(x), ws)
    with pytest.raises(ValueError):
        ctx.chunk_attention(pool, 1, crf.Chunks([t], [2], [0]), x, torch.zeros_like(x), ws)
    with pytest.raises(ValueError):
        ctx.pages_fork(pool, t, crf.PageTables([t], [16], [t]), ws)
    with pytest.raises(ValueError):
        ctx.pages_release(t, crf.PageTables([t], [16]), ws)


def test_heads_marshalling():
    buf = ctypes.create_string_buffer(2 * crf._HEADS)

    def put(x, out, dim=64, device=-1):
        n = crf._put_heads(buf, crf._HEADS, device, "x", x, out, dim)
        h = abi.Heads.from_buffer(buf, crf._HEADS)
        assert n == h.heads
        return h.x, h.out, h.heads, h.x_row, h.x_head, h.out_row, h.out_head

    x = torch.zeros(5, 7, 64, dtype=torch.bfloat16)[:, 1:4]
    y = torch.zeros(3, 5, 64, dtype=torch.bfloat16).transpose(0, 1)
    assert put(x, None) == (x.data_ptr(), None, 3, 448, 64, 0, 0)
    assert put(x, x) == (x.data_ptr(), x.data_ptr(), 3, 448, 64, 448, 64)
    assert put(x, y) == (x.data_ptr(), y.data_ptr(), 3, 448, 64, 64, 320)
    z = torch.zeros(2, 3, 128, dtype=torch.bfloat16)[..., ::2]
    for bad in ((x, None, 32), (x, None, 64, 0), (z, None), (x, torch.zeros(5, 3, 64)), (x, y[:4]), (x[0], None),
                (torch.zeros(2, 3, 64, dtype=torch.bfloat16), z)):
        with pytest.raises(ValueError):
            put(*bad)
