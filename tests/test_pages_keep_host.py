"""Rows taken back from page tables without a GPU: what the entry point refuses."""
import pytest

import paper_2604_02570_amd as W
from test_dense_f8_host import pool
from test_dense_host import A, ctx, refuses  # noqa: F401


def keep(ctx, p=None, **kw):
    a = {**dict(kept=A, lens=A, n_free=A, lens_out=A, n_free_out=A), **kw}
    W.wsvd_pages_keep(ctx, p or pool(), a["kept"], a["lens"], a["n_free"], a["lens_out"], a["n_free_out"], 0)


def test_page_pools_refused(ctx):
    for kw, status in ((dict(table=None), W.E_NULL), (dict(free=None), W.E_NULL), (dict(batch=0), W.E_SHAPE), (dict(batch=65537), W.E_SHAPE),
                       (dict(page_rows=24), W.E_SHAPE), (dict(max_pages=0), W.E_SHAPE), (dict(n_pages=0), W.E_SHAPE), (dict(n_pages=(1 << 24) + 1), W.E_SHAPE),
                       (dict(page_rows=4096, max_pages=1 << 16), W.E_SHAPE), (dict(table=A + 2), W.E_ALIGN), (dict(free=A + 1), W.E_ALIGN)):
        refuses(status, keep, ctx, pool(**kw))


@pytest.mark.parametrize("name", ["kept", "lens", "n_free", "lens_out", "n_free_out"])
def test_arguments_refused(ctx, name):
    refuses(W.E_NULL, keep, ctx, **{name: None})
    refuses(W.E_ALIGN, keep, ctx, **{name: A + 2})
    refuses(W.E_NULL, keep, None)
