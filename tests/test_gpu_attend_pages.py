"""Page ids outside the cache: the rows that see a key of such a page are NaN, all others are as without it, whichever
tiles and workgroups they share.  Bounds as in test_gpu_attend."""
import numpy as np
import pytest
import torch

import paper_2609_14636_amd as P
from tests.test_gpu_attend import BF, F32, check, make, run

pytestmark = pytest.mark.gpu


def spoil_and_check(x, s, page_no, bad_id):
    """Entry page_no of sequence s's table is bad_id."""
    page = x["k"].shape[1]
    good = int(x["table"][s, page_no])
    x["table"][s, page_no] = bad_id
    o, lse, flags = run(x)
    assert int(flags) == P.STRIDE_FLAG_BAD_PAGE
    x["table"][s, page_no] = good
    lost = np.zeros(len(o), bool)
    ctx, n = x["ctxs"][s], x["n"][s]
    for slot in range(page_no * page, min((page_no + 1) * page, ctx + n)):
        for i in range(n):
            lost[x["offs"][s] + i] |= slot < ctx or bool(x["sees"](s, i, slot - ctx))
    at = torch.from_numpy(lost).cuda()
    assert bool(o[at].isnan().all()) and bool(lse[at].isnan().all())
    assert 0 < lost.sum() < len(lost)
    check(x, o, lse, np.flatnonzero(~lost))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n,ctx", [([3, 5], [40, 64 * 3 - 4]), ([6, 13], [7, 64 - 12]), ([2, 150], [1000, 33]), ([70, 40], [5, 640 - 39])])
def test_a_page_of_new_tokens(dtype, d, page, n, ctx):
    """The last page of a chain, whose keys only its last rows see; few rows and many, whole blocks per page and not."""
    x = make(dtype, 4, 2, d, page, n, ctx, by_head=d == 96, seed=d + page)
    last = (n[1] + ctx[1] - 1) // page
    for bad in (x["k"].shape[0], -1):
        spoil_and_check(x, 1, last, bad)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [8, 32, 64])
@pytest.mark.parametrize("n,ctx", [([4, 30], [9, 50]), ([4, 90], [9, 2000]), ([66, 90], [300, 31])])
def test_a_page_in_the_middle_of_a_tree(dtype, page, n, ctx):
    x = make(dtype, 6, 2, 64, page, n, ctx, tree="tree", seed=page)
    spoil_and_check(x, 1, (ctx[1] + n[1] // 2) // page, 1 << 30)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n", [[1, 2, 1], [40, 60, 1]])
def test_a_cached_page(dtype, page, n):
    """All rows of its sequence see it, also those of a sequence that many workgroups share."""
    x = make(dtype, 4, 1, 128, page, n, [100, 9000, 64], seed=3)
    spoil_and_check(x, 1, 4000 // page, x["k"].shape[0])


@pytest.mark.parametrize("dtype,n,ctx,page", [(BF, 8, 8, 4), (BF, 8, 28, 32), (BF, 40, 24, 16), (BF, 40, 44, 64), (F32, 20, 16, 16),
                                              (F32, 20, 48, 64)])
def test_a_page_that_no_row_sees(dtype, n, ctx, page):
    """Its id is reported; nothing is NaN."""
    x = make(dtype, 4, 2, 64, page, [n], [ctx], tree=lambda s, i, j: j == i and j < 4, seed=1)
    last = (n + ctx - 1) // page
    assert last * page >= ctx + 4
    good = int(x["table"][0, last])
    x["table"][0, last] = -7
    o, lse, flags = run(x)
    assert int(flags) == P.STRIDE_FLAG_BAD_PAGE
    x["table"][0, last] = good
    check(x, o, lse)
