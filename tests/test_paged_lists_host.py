"""Attention over lists of rows of a cache in pages: lists, counts and sums of another type, shape or order than the kernel reads are refused.
Host only."""
import types

import pytest
import torch

from paper_2503_07518_amd import binding as tb

B, Hq, Hkv, D, CAP = 3, 8, 2, 64, 12
INT, BF16 = torch.int32, torch.bfloat16


@pytest.fixture
def call(monkeypatch):
    """The call with some arguments replaced; returns what the library gets."""
    seen = []
    monkeypatch.setattr(tb, "_lib", types.SimpleNamespace(tb_sparse_decode_attn_paged=lambda *a: seen.append(a) or 0))
    monkeypatch.setattr(tb, "_stream_on", lambda *a: 0)
    pages = torch.zeros((9, Hkv, 16, D), dtype=BF16)
    cache = tb.PagedCache(pages, pages.clone(), torch.zeros((B, 4), dtype=INT))
    desc = tb.make_paged_desc(64, Hq, cache)

    def run(**kw):
        seen.clear()
        args = dict(q=torch.zeros((B, Hq, D), dtype=BF16), idx=torch.zeros((B, Hq, CAP), dtype=INT), count=torch.zeros((B, Hq), dtype=INT), max_count=CAP,
                    sm_scale=1.0, out=torch.zeros((B, Hq, D)), lse=torch.zeros((B, Hq)), ws=torch.zeros(256, dtype=torch.uint8))
        tb.tb_sparse_decode_attn_paged(desc, cache, **dict(args, **kw))
        return seen[0]
    return run


def test_taken(call):
    assert call()[5:7] == (CAP, CAP)  # (idx_cap, max_count)
    assert call(lse=None)[11] is None
    wide = torch.zeros((B, Hq, 2 * CAP), dtype=INT)
    assert call(idx=wide[..., :CAP])[5:7] == (2 * CAP, CAP)
    assert call(idx=wide, max_count=CAP + 5)[5:7] == (2 * CAP, CAP + 5)
    assert call(idx=torch.zeros((B, Hq, 0), dtype=INT), max_count=0)[6] == 0


@pytest.mark.parametrize("bad", [
    dict(idx=torch.zeros((B, Hq, CAP), dtype=torch.int64)), dict(idx=torch.zeros((B, Hq, CAP))), dict(idx=torch.zeros((B, Hkv, CAP), dtype=INT)),
    dict(idx=torch.zeros((2, Hq, CAP), dtype=INT)), dict(idx=torch.zeros((B * Hq, CAP), dtype=INT)), dict(idx=torch.zeros((B, Hq, 2 * CAP), dtype=INT)[..., ::2]),
    dict(idx=torch.zeros((Hq, B, CAP), dtype=INT).transpose(0, 1)), dict(idx=torch.zeros((B, 2 * Hq, CAP), dtype=INT)[:, :Hq]),
    dict(idx=torch.zeros((B, Hq, CAP - 1), dtype=INT)), dict(idx=torch.zeros((B, Hq, 2 * CAP), dtype=INT)[..., :CAP - 1]),
    dict(count=torch.zeros((B, Hq), dtype=torch.int64)), dict(count=torch.zeros((B, Hkv), dtype=INT)), dict(count=torch.zeros((Hq, B), dtype=INT).t()),
    dict(count=torch.zeros((B, Hq, 1), dtype=INT)), dict(lse=torch.zeros((B, Hq), dtype=torch.float64)), dict(lse=torch.zeros((B, Hkv))), dict(lse=torch.zeros((Hq, B)).t()),
])
def test_refused(call, bad):
    with pytest.raises(AssertionError):
        call(**bad)
