"""The page tables' calls report a free list's length that is none, and take the nearest that is."""
import pytest
import torch

import paper_2604_02570_amd as W

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("call", ["grow", "release", "keep"])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("batch", [2, 300])
@pytest.mark.parametrize("n_free,taken", [(-1, 0), (-2 ** 31, 0), (41, 40), (2 ** 31 - 1, 40), (40, 40), (0, 0)])
def test_a_free_list_of_no_length(call, in_place, batch, n_free, taken):
    """Nothing is to be grown or given back: the list's length alone is wrong."""
    ctx, R, P, pages = W.wsvd_create(0), 16, 300, 40
    table, free, lens, count = torch.full((batch, P), -1, dtype=torch.int32, device="cuda"), torch.arange(pages, dtype=torch.int32, device="cuda"), ints([0] * batch), ints([n_free])
    pool = W.make_page_pool(table, free, batch, R, P, pages)
    lens_out, count_out = (lens, count) if in_place else (torch.full_like(lens, 7), torch.full_like(count, 7))
    if call == "grow":
        W.wsvd_pages_grow(ctx, pool, ints([0] * batch), 5000, lens, count, lens_out, count_out)
    else:
        getattr(W, "wsvd_pages_" + call)(ctx, pool, ints([1] * batch), lens, count, lens_out, count_out)
    status = W.wsvd_check(ctx)
    W.wsvd_destroy(ctx)
    assert count_out.tolist() == [taken] and lens_out.tolist() == [0] * batch
    assert status == (0 if n_free == taken else W.E_SHAPE)
