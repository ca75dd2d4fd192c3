"""Attention over lists in a pool of pages as large as it takes, and over lists as long as its non-temporal loads ask for."""
import math

import pytest
import torch

from paper_2503_07518_amd import binding as tb
from paged_util import make
from test_gpu_paged import BF, DEV, lists, on_gpu, run_sparse

pytestmark = pytest.mark.gpu


def test_a_pool_of_64_GiB():
    """One KV head, K and V of a page side by side, rows in the last pages: the bits of a small pool's."""
    c = on_gpu(make(BF, 8, 1, 128, 64, [0, 0], [600, 739], seed=8))
    q = torch.randn((2, 8, 128), generator=c.gen).to(BF)
    idx, count = lists(c, 300)
    want = run_sparse(c, q, idx, count, 300, (590, 600), 0.09)
    pages = (1 << 36) // (2 * 64 * 128 * 2)
    pool = torch.empty((pages, 2, 64, 128), dtype=BF, device=DEV)
    few = c.K.shape[0]
    pool[0] = math.nan
    pool[-few:, 0], pool[-few:, 1] = c.K[:, 0].to(DEV), c.V[:, 0].to(DEV)
    c.cache = tb.PagedCache(pool[:, :1], pool[:, 1:], (c.table + (pages - few)).to(DEV))
    for got, x in zip(run_sparse(c, q, idx, count, 300, (590, 600), 0.09), want):
        assert torch.equal(got, x) and bool(torch.isfinite(got).all())
    c.cache = None
    del pool
    torch.cuda.empty_cache()
