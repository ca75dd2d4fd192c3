"""What the interval loop over a 4-bit cache refuses, before anything is launched: tensors of another type or shape than the one it was
made for, which the kernels would read past their end or as other numbers."""
import pytest
import torch

from paper_2503_07518_amd import binding as tb
from paper_2503_07518_amd.interval import MxIntervalDecoder

F32, BF16 = torch.float32, torch.bfloat16
B, Hkv, Hq, D, d, N, P = 2, 2, 8, 64, 32, 40, 4


@pytest.fixture(autouse=True)
def no_launches(monkeypatch):
    """Workspaces in host memory, nothing to clear them with; whatever launches a kernel is an error."""
    def launched(*a, **k):
        raise RuntimeError("launched")
    monkeypatch.setattr(tb, "new_workspace", lambda *a, **k: torch.zeros(256, dtype=torch.uint8))
    for name in ("tb_quantize_mx", "tb_score_mx", "tb_select_topk", "tb_expand_neighbors", "tb_sparse_decode_attn_mx", "tb_sparse_decode_attn_shared_mx",
                 "tb_project_keys"):
        monkeypatch.setattr(tb, name, launched)


def loop(W=None, dtype=BF16, headless=False, Kimp=d):
    cache = tb.MxCache(B, Hkv, N, D, Kimp, device="cpu")
    if headless:
        cache.Kimp = tb.MxCache(B, 1, N, D, Kimp, device="cpu").Kimp
    W = torch.zeros((1, D, d), dtype=dtype) if W is None and not headless else W
    return MxIntervalDecoder(cache, W, Hq, 4, P, 1, headless=headless, dtype=dtype)


@pytest.mark.parametrize("kw", [dict(W=torch.zeros((1, D, d))), dict(W=torch.zeros((1, D, d), dtype=BF16), dtype=F32),
                                dict(W=torch.zeros((1, 2 * D, d), dtype=BF16)), dict(W=torch.zeros((1, D, 2 * d), dtype=BF16)), dict(Kimp=2 * d), dict(W=torch.zeros((D, d), dtype=BF16))])
def test_projections_of_another_type_or_shape(kw):
    with pytest.raises(AssertionError):
        loop(**kw)


@pytest.mark.parametrize("headless", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_queries_of_another_type_or_shape(dtype, headless):
    other = BF16 if dtype == F32 else F32
    Hl = 1 if headless else Hq
    x = loop(dtype=dtype, headless=headless)
    q, q_imp = torch.zeros((B, Hq, D), dtype=dtype), torch.zeros((B, Hl, d), dtype=dtype)
    for bad in ((q.to(other), q_imp), (q, q_imp.to(other)), (q[:1], q_imp), (q[:, :4], q_imp), (q[..., :32], q_imp), (q, q_imp[..., :16]), (q, q_imp[:1]),
                (q, torch.zeros((B, Hl + 1, d), dtype=dtype))):
        with pytest.raises(AssertionError):
            x.step(0, *bad)
    with pytest.raises(RuntimeError, match="launched"):
        x.step(0, q, q_imp)


def test_rows_of_another_type_or_shape():
    x = loop()
    rows = torch.zeros((B, Hkv, 3, D), dtype=BF16)
    for bad in ((rows.float(), rows.float()), (rows, rows[:, :, :2]), (rows[:, :1], rows[:, :1]), (rows[..., :32], rows[..., :32])):
        with pytest.raises(AssertionError):
            x.append(*bad)
    with pytest.raises(ValueError):
        x.append(*[torch.zeros((B, Hkv, N + 1, D), dtype=BF16)] * 2)
    assert x.N == 0
    with pytest.raises(RuntimeError, match="launched"):
        x.append(rows, rows)
    assert x.N == 0 and x.n_waiting == 0
