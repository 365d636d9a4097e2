"""Calls on normed heads and on rows of logits, as far as they go without a GPU: struct layouts, the C ABI's refusals (made before
the context's device is touched, so a zeroed stand-in serves as the context) and the binding's own checks."""
import ctypes
import math
import shutil
import subprocess

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300 import abi
from tests.test_extend_host import A16, HEADER, chunks, ctx, heads, lib, pool, ref, rope  # noqa: F401

EINVAL, ESHAPE, EUNSUPPORTED, ENOMEM = abi.EINVAL, abi.ESHAPE, abi.EUNSUPPORTED, abi.ENOMEM


def test_struct_layout_and_limits_match_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    (tmp_path / "l.c").write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{HEADER}"\nint main(void){{printf("%zu %zu %zu %d %d", '
                                  "sizeof(crf_norm), offsetof(crf_norm, gain), offsetof(crf_norm, eps), CRF_MAX_TOP, CRF_MAX_VOCAB);return 0;}")
    subprocess.run([cc, str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [ctypes.sizeof(abi.Norm), abi.Norm.gain.offset, abi.Norm.eps.offset, abi.MAX_TOP, abi.MAX_VOCAB]


def norms(*n):
    return (abi.Norm * 2)(*(abi.Norm(*x) for x in (n or ((A16, 1e-6), (A16, 1e-6)))))


def call_norm(lib, ctx, r=None, p=None, n=None, n_parts=1, type=abi.BF16, rows=3, positions=A16):  # noqa: F811
    return lib.crf_norm_rotary(ctx, ref(r or rope()), (abi.Heads * 2)(*(p or (heads(), heads()))), n or norms(), n_parts, type, rows,
                               positions, None)


def call_grad(lib, ctx, r=None, p=None, n=None, g=None, dg=(A16, A16), n_parts=1, type=abi.BF16, rows=3, positions=A16,  # noqa: F811
              ws=A16, ws_bytes=1 << 30):
    return lib.crf_norm_rotary_grad(ctx, ref(r or rope()), (abi.Heads * 2)(*(p or (heads(), heads()))), n or norms(),
                                    (abi.Heads * 2)(*(g or (heads(x=A16 + 8192), heads(x=A16 + 8192)))),
                                    None if dg is None else (ctypes.c_void_p * 2)(*dg), n_parts, type, rows, positions, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [call_norm, call_grad])
def test_norm_refusals(lib, ctx, call):  # noqa: F811
    for kw, status in [(dict(rot_dim=63), EUNSUPPORTED), (dict(head_dim=258, rot_dim=2), EUNSUPPORTED), (dict(theta=0.0), EINVAL)]:
        assert call(lib, ctx, r=rope(**kw)) == status
    for kw, status in [(dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(heads=0), EINVAL), (dict(x_row=-1), EINVAL), (dict(x=A16 + 1), EINVAL),
                       (dict(out_row=0), ESHAPE), (dict(out_head=32), ESHAPE), (dict(x=A16, out=A16, x_row=512), ESHAPE)]:
        assert call(lib, ctx, p=(heads(**kw), heads())) == status
        assert call(lib, ctx, p=(heads(), heads(**kw)), n_parts=2) == status
    for bad in ((None, 1e-6), (A16 + 1, 1e-6), (A16, -1e-6), (A16, math.nan), (A16, math.inf)):
        assert call(lib, ctx, n=norms(bad, (A16, 0.0))) == EINVAL
        assert call(lib, ctx, n=norms((A16, 0.0), bad), n_parts=2) == EINVAL
    assert call(lib, ctx, n=norms((A16 + 2, 0.0), (A16, 0.0)), type=abi.FP32) == EINVAL
    assert call(lib, ctx, n_parts=0) == EINVAL and call(lib, ctx, n_parts=3) == EINVAL
    assert call(lib, ctx, type=3) == EUNSUPPORTED and call(lib, ctx, rows=-1) == EINVAL
    assert call(lib, ctx, positions=None) == EINVAL and call(lib, ctx, positions=A16 + 2) == EINVAL
    assert call(lib, None) == EINVAL


def test_norm_of_no_rows_is_nothing(lib, ctx):  # noqa: F811
    assert call_norm(lib, ctx, rows=0, positions=None) == abi.OK
    assert lib.crf_norm_rotary(ctx, ref(rope()), ref(heads()), None, 1, 0, 3, A16, None) == EINVAL


def test_gradient_refusals(lib, ctx):  # noqa: F811
    other = heads(x=A16 + 8192)
    for kw, status in [(dict(x=None), EINVAL), (dict(heads=3), ESHAPE), (dict(x=A16 + 1), EINVAL), (dict(x_head=-64), EINVAL)]:
        assert call_grad(lib, ctx, g=(heads(**{**dict(x=A16 + 8192), **kw}), other)) == status
        assert call_grad(lib, ctx, g=(other, heads(**{**dict(x=A16 + 8192), **kw})), n_parts=2) == status
    # over the gradient, with other strides
    assert call_grad(lib, ctx, g=(heads(x=A16 + 4096, x_row=512), other)) == ESHAPE
    assert call_grad(lib, ctx, dg=None) == EINVAL and call_grad(lib, ctx, dg=(None, A16)) == EINVAL
    assert call_grad(lib, ctx, dg=(A16, A16 + 2), n_parts=2) == EINVAL
    assert call_grad(lib, ctx, ws=None) == EINVAL and call_grad(lib, ctx, ws=A16 + 16) == EINVAL and call_grad(lib, ctx, ws_bytes=64) == ENOMEM
    n = ctypes.c_size_t()
    assert lib.crf_norm_rotary_workspace_size(ctx, 64, 3, ctypes.byref(n)) == abi.OK and n.value % 256 == 0 and n.value >= 3 * 64 * 4
    assert call_grad(lib, ctx, ws=A16 + 16, ws_bytes=n.value) == EINVAL
    for dim, rows, status in ((1, 3, EUNSUPPORTED), (257, 3, EUNSUPPORTED), (64, -1, EINVAL)):
        assert lib.crf_norm_rotary_workspace_size(ctx, dim, rows, ctypes.byref(n)) == status
    assert lib.crf_norm_rotary_workspace_size(ctx, 64, 3, None) == EINVAL


def test_normed_append_refusals(lib, ctx):  # noqa: F811
    def call(r=True, q=None, qn=None, k=None, kn=(A16, 1e-6), hkv=2, d=64, ch=((3, 5, 8, A16),)):
        one = lambda n: None if n is None else ref(abi.Norm(*n))  # noqa: E731
        return lib.crf_cache_append_normed(ctx, ref(rope()) if r else None, ref(pool()), 0, hkv, d, chunks(*ch), len(ch),
                                           None if q is None else ref(q), one(qn), ref(k or heads(heads=2)), one(kn), ref(heads(heads=2)), None)

    assert call(r=False) == EINVAL and call(kn=None) == EINVAL and call(q=heads()) == EINVAL
    assert call(kn=(None, 1e-6)) == EINVAL and call(kn=(A16, -1.0)) == EINVAL and call(q=heads(), qn=(A16 + 1, 0.0)) == EINVAL
    assert call(k=heads(heads=3)) == ESHAPE and call(d=128) == ESHAPE and call(d=96) == EUNSUPPORTED
    assert call(ch=((1, 0, 1, None),)) == EINVAL
    assert call(ch=((0, 0, 0, None),)) == abi.OK


def call_logprobs(lib, ctx, z=A16, type=abi.FP32, rows=3, vocab=100, stride=100, t=A16, lp=A16, h=A16, lse=A16, k=5, ids=A16, tops=A16):  # noqa: F811
    return lib.crf_logprobs(ctx, z, type, rows, vocab, stride, t, lp, h, lse, k, ids, tops, None)


def call_logprobs_grad(lib, ctx, z=A16, type=abi.FP32, rows=3, vocab=100, stride=100, t=A16, lse=A16, h=A16, g=A16, gh=A16,  # noqa: F811
                       dz=A16 + 65536, dstride=100):
    return lib.crf_logprobs_grad(ctx, z, type, rows, vocab, stride, t, lse, h, g, gh, dz, dstride, None)


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), EINVAL), (dict(z=A16 + 2), EINVAL), (dict(type=3), EUNSUPPORTED), (dict(type=-1), EUNSUPPORTED), (dict(rows=-1), EINVAL),
    (dict(rows=(1 << 24) + 1), EUNSUPPORTED), (dict(vocab=0), EUNSUPPORTED), (dict(vocab=(1 << 20) + 1, stride=1 << 21), EUNSUPPORTED),
    (dict(stride=99), ESHAPE), (dict(stride=-100), ESHAPE), (dict(stride=(1 << 40) + 1), ESHAPE), (dict(t=A16 + 2), EINVAL), (dict(lse=A16 + 1), EINVAL),
    (dict(h=A16 + 2), EINVAL),
])
def test_logprobs_refusals(lib, ctx, kw, status):  # noqa: F811
    assert call_logprobs(lib, ctx, **kw) == status
    assert call_logprobs_grad(lib, ctx, **kw) == status


def test_logprobs_refusals_of_their_own(lib, ctx):  # noqa: F811
    for kw, status in [(dict(k=-1), EUNSUPPORTED), (dict(k=33), EUNSUPPORTED), (dict(vocab=4), EUNSUPPORTED), (dict(t=None), EINVAL),
                       (dict(ids=None, tops=None), EINVAL), (dict(ids=A16 + 2), EINVAL), (dict(tops=A16 + 1), EINVAL), (dict(lp=A16 + 2), EINVAL)]:
        assert call_logprobs(lib, ctx, **kw) == status
    assert call_logprobs(lib, None) == EINVAL and call_logprobs_grad(lib, None) == EINVAL
    assert call_logprobs(lib, ctx, rows=0, z=None) == abi.OK and call_logprobs_grad(lib, ctx, rows=0, z=None) == abi.OK
    for kw, status in [(dict(dz=None), EINVAL), (dict(dz=A16 + 2), EINVAL), (dict(dstride=99), ESHAPE), (dict(lse=None), EINVAL), (dict(t=None), EINVAL),
                       (dict(h=None), EINVAL), (dict(g=A16 + 2), EINVAL), (dict(gh=A16 + 2), EINVAL), (dict(dz=A16, dstride=104), ESHAPE)]:
        assert call_logprobs_grad(lib, ctx, **kw) == status


def test_binding_checks(lib):  # noqa: F811
    """What the binding refuses before the library is called (tensors of the host)."""
    c = crf.Context.__new__(crf.Context)
    c.lib, c.h, c.device = None, None, -1  # the host's tensors are on device -1
    c._parts, c._norms, c._dgains = ctypes.create_string_buffer(1024), ctypes.create_string_buffer(64), (ctypes.c_void_p * 2)()
    r = crf.Rope(64)
    x, w, pos = torch.zeros(3, 2, 64), torch.zeros(64), torch.zeros(3, dtype=torch.int32)
    ws = torch.zeros(256, dtype=torch.uint8)

    def refuses(f, *a, **kw):
        with pytest.raises(ValueError):
            f(*a, **kw)

    refuses(c.norm_rotary, r, pos, x.double(), w)
    refuses(c.norm_rotary, r, pos[:2], x, w)
    refuses(c.norm_rotary, r, pos, x[..., :32], w)
    refuses(c.norm_rotary, r, pos, x, w[:32])
    refuses(c.norm_rotary, r, pos, x, w.half())
    refuses(c.norm_rotary, r, pos, x, torch.zeros(128)[::2])
    refuses(c.norm_rotary, r, pos, x, w, k=x)
    refuses(c.norm_rotary, r, pos, x, w, k=x.half(), k_gain=w.half())
    refuses(c.norm_rotary_grad, r, pos, x, w, x, x, w, ws, k=x, k_gain=w)
    refuses(c.norm_rotary_grad, r, pos, x, w, x[:2], x, w, ws)
    refuses(c.norm_rotary_grad, r, pos, x, w, x.half(), x, w, ws)
    refuses(c.norm_rotary_grad, r, pos, x, w, x, x, w[:32], ws)
    refuses(c.norm_rotary_grad, r, pos, x, w, x, x, w.half(), ws)
    z, f, i = torch.zeros(3, 50), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    refuses(c.logprobs, z.double())
    refuses(c.logprobs, z[0])
    refuses(c.logprobs, torch.zeros(50, 3).t())
    refuses(c.logprobs, z, i.long())
    refuses(c.logprobs, z, i[:2])
    refuses(c.logprobs, z, i, logprob=f.half())
    refuses(c.logprobs, z, i, lse=torch.zeros(6)[::2])
    refuses(c.logprobs, z, i, top_ids=torch.zeros(3, 4))
    refuses(c.logprobs, z, i, top_ids=torch.zeros(3, 4, dtype=torch.int32), top_logprobs=torch.zeros(3, 5))
    refuses(c.logprobs_grad, z, i, None, z)
    refuses(c.logprobs_grad, z, i, f, z.half())
    refuses(c.logprobs_grad, z, i, f, z[:, :40])
    refuses(c.logprobs_grad, z, i, f, z, g_logprob=f[:2])
    c.h = ctypes.c_void_p()
