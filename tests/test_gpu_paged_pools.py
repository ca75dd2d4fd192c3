"""Attention over lists in a pool of pages as large as it takes, and over lists as long as its non-temporal loads ask for."""
import math
import types

import pytest
import torch

from oracle import paged as ref
from paper_2503_07518_amd import binding as tb
from paged_util import attn_bounds, close, make
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


def test_lists_that_are_not_kept():
    """Rows of a batch that few heads list and no cache holds, read non-temporally: the bits of the call over a contiguous cache; with holes,
    sampled heads against 64 bits."""
    B, Hq, Hkv, D, page, n, k = 16, 32, 8, 128, 64, 16384, 2048
    tail, scale = (n - 7, n), D ** -0.5
    distinct = n * (1 - (1 - (k + 7) / n) ** (Hq // Hkv))
    assert B * Hkv * distinct * 2 * D * 2 >= 375e6 and (Hq // Hkv) * (k + 7) <= 1.4 * distinct
    gen = torch.Generator(device=DEV).manual_seed(3)
    entries = n // page
    pages = B * entries + 3
    table = torch.randperm(pages, generator=gen, device=DEV)[:B * entries].view(B, entries).to(torch.int32)
    K, V = (torch.randn((pages, Hkv, page, D), generator=gen, device=DEV, dtype=BF) for _ in range(2))
    q = torch.randn((B, Hq, D), generator=gen, device=DEV).to(BF)
    idx = torch.rand((B, Hq, n - 7), generator=gen, device=DEV).topk(k, dim=-1).indices.sort(-1).values.to(torch.int32)
    count = torch.randint(0, k + 1, (B, Hq), generator=gen, device=DEV).to(torch.int32)
    count[0], count[1, 0] = k, 0

    def paged(table):
        cache = tb.PagedCache(K, V, table)
        d = tb.make_paged_desc(n, Hq, cache)
        out, lse = torch.full((B, Hq, D), 7.0, device=DEV), torch.full((B, Hq), 7.0, device=DEV)
        tb.tb_sparse_decode_attn_paged(d, cache, q, idx, count, k, scale, out, lse, tb.new_workspace(tb.TB_OP_ATTN, d, k + 7), *tail)
        return out, lse

    out, lse = paged(table)
    Kc, Vc = (x[table.long()].transpose(1, 2).reshape(B, Hkv, n, D) for x in (K, V))
    d = tb.make_desc(n, Hq, K=Kc, V=Vc)
    o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
    tb.tb_sparse_decode_attn(d, q, Kc, Vc, idx, count, k, scale, o2, l2, tb.new_workspace(tb.TB_OP_ATTN, d, k + 7), *tail)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    del Kc, Vc
    # a tenth of the pages are gone, and those behind the last one
    holed = table.clone()
    gone = torch.rand(table.shape, generator=gen, device=DEV) < 0.1
    gone[2, -1] = True
    holed[gone] = torch.tensor([-1, pages, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV).repeat(B * entries // 4 + 1)[:int(gone.sum())]
    out, lse = paged(holed)
    c = types.SimpleNamespace(D=D, dtype=BF)
    for b in (0, 1, 2, 9):
        for h in (0, 5, 31):
            rows = torch.cat((idx[b, h, :int(count[b, h])].long(), torch.arange(*tail, device=DEV)))
            rows = rows[~gone[b, rows // page]]
            at = table[b, rows // page].long()
            want, l, mag = ref.attend(q[b, h].double().cpu(), K[at, h * Hkv // Hq, rows % page].double().cpu(), V[at, h * Hkv // Hq, rows % page].double().cpu(), rows, scale)
            tol, tol_lse = attn_bounds(c, q[b, h].cpu(), K[at, h * Hkv // Hq, rows % page].cpu(), V, k + 7, scale, mag, want, exact_weights=True) if len(rows) else (0, 0)
            close(out[b, h], want, tol + mag * 16 * 2.0 ** -24)
            close(lse[b, h], torch.tensor(l), tol_lse + abs(l) * 2.0 ** -22 if len(rows) else 0)
