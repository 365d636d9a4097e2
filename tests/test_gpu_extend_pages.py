"""Page calls at the ends of their ranges, exact like those of test_gpu_extend.py."""
import pytest
import torch

import paper_2609_30884_gb300 as crf
from tests.test_gpu_extend import Pool, assert_rejected, compact_model, fork_model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = crf.Context(0)
    yield c
    c.close()


def assert_forked(ctx, s, deep):
    tables, outs = s.page_tables()
    want, refs, k, v = fork_model([t.tolist() for t in s.tables], s.tokens, s.refs.tolist(), s.k, s.v, deep)
    ctx.pages_fork(s.pool, s.refs, tables, ctx.pages_workspace(s.total, tables), deep=deep)
    ctx.check()
    assert [o.tolist() for o in outs] == want and s.refs.tolist() == refs and torch.equal(s.k, k) and torch.equal(s.v, v)


def test_fork_rejects_counts_without_room(ctx):
    """A count that the call's entries could take past the largest int32 would come out negative."""
    s = Pool(71, [100, 40], 20, layers=2)
    tables, outs = s.page_tables()
    ws = ctx.pages_workspace(s.total, tables)
    entries, page = 7 + 3, int(s.tables[0][2])
    for count in (2**31 - 1, 2**31 - entries):
        s.refs[page] = count
        assert_rejected(ctx, s, lambda: ctx.pages_fork(s.pool, s.refs, tables, ws), "EINVAL", outs)
    assert_forked(ctx, s, deep=True)  # raises no count
    s.refs[page] = 2**31 - 1 - entries
    assert_forked(ctx, s, deep=False)


# (heads, head size, layers): units of a page cut by 16 KB, the last one shorter; whole units; more layers than one copy
# launch takes
SHAPES = [(5, 128, 2), (8, 128, 2), (9, 64, 2), (17, 64, 1), (1, 64, 65), (2, 128, 130)]


@pytest.mark.parametrize("deep", [False, True])
@pytest.mark.parametrize("hkv,dim,layers", SHAPES)
def test_fork_copies_pages_of_any_shape(ctx, hkv, dim, layers, deep):
    assert_forked(ctx, Pool(72, [41, 16, 1, 0, 77], 14, layers=layers, hkv=hkv, dim=dim), deep)


@pytest.mark.parametrize("hkv,dim,layers", SHAPES)
def test_compact_copies_pages_of_any_shape(ctx, hkv, dim, layers):
    s = Pool(73, [41, 16, 1, 0, 77], 14, layers=layers, hkv=hkv, dim=dim)
    want, refs, k, v = compact_model([t.tolist() for t in s.tables], s.refs.tolist(), s.k, s.v)
    tables, outs = s.page_tables()
    assert [t.tolist() for t in s.tables] != want  # something moves
    ctx.pages_compact(s.pool, s.refs, tables, ctx.pages_workspace(s.total, tables))
    ctx.check()
    assert [o.tolist() for o in outs] == want and s.refs.tolist() == refs and torch.equal(s.k, k) and torch.equal(s.v, v)
