"""One place for two gains' gradients: each part writes its own sum, so the call is refused (also where q and k share their gain)."""
import pytest

from paper_2609_30884_gb300 import abi
from tests.test_extend_host import A16, ctx, heads, lib, ref, rope  # noqa: F401
from tests.test_normed_host import call_grad


@pytest.mark.parametrize("rows", [0, 3])
def test_gradients_of_two_gains_in_one_place_are_refused(lib, ctx, rows):  # noqa: F811
    assert call_grad(lib, ctx, dg=(A16, A16), n_parts=2, rows=rows) == abi.EINVAL
    assert b"dgains overlap" in lib.crf_last_error()
    # parts of one array that do not reach into each other are not that: refused for the workspace alone
    assert call_grad(lib, ctx, dg=(A16, A16 + 64 * 4), n_parts=2, rows=3, ws_bytes=64) == abi.ENOMEM
    for near in (A16 + 4, A16 + 63 * 4):
        assert call_grad(lib, ctx, dg=(A16, near), n_parts=2, rows=rows, ws_bytes=64) == abi.EINVAL
        assert call_grad(lib, ctx, dg=(near, A16), n_parts=2, rows=rows, ws_bytes=64) == abi.EINVAL
    assert call_grad(lib, ctx, dg=(A16, A16), n_parts=1, rows=3, ws_bytes=64) == abi.ENOMEM
