"""The interval loop over a cache in pages: the same bits as the loop over a contiguous cache with the same rows, and prompts against 64 bits."""
import pytest
import torch

from oracle import paged as ref
from paper_2503_07518_amd import binding as tb
from paper_2503_07518_amd.interval import IntervalDecoder, PagedIntervalDecoder
from paged_util import attn_bounds, close, half_step, make

pytestmark = pytest.mark.gpu
DEV = "cuda"
P = 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mode,expand", [(0, False), (1, False), (0, True)])
def test_loop(dtype, mode, expand):
    B, Hq, Hkv, D, d = 2, 8, 2, 64, 16
    total = 260
    c = make(dtype, Hq, Hkv, D, 16, [total] * B, [0] * B, seed=4)
    cache = tb.PagedCache(torch.full_like(c.K, float("nan"), device=DEV), torch.full_like(c.V, float("nan"), device=DEV), c.table.to(DEV))
    q, k, v = (x.view(B, total, -1, D).to(DEV) for x in (c.q, c.k, c.v))
    W = (torch.randn((1, D, d), generator=c.gen) / 8).to(dtype).to(DEV)
    q_imp = torch.randn((total, B, Hq, d), generator=c.gen).to(dtype).to(DEV)
    f = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
    kw = dict(Hq=Hq, k=30, P=P, radius=1, sink=2, window=3, sm_scale=D ** -0.5, mode=mode, expand_on_predict=expand)
    loop = PagedIntervalDecoder(cache, W, inv_freq=f, **kw)
    Ncap = loop.Ncap
    K, V, Kimp = (torch.zeros((B, Hkv, Ncap, n), dtype=dtype, device=DEV) for n in (D, D, d))
    flat = None

    def contiguous():
        rows = torch.arange(loop.N, device=DEV)
        at = cache.table[:, rows // 16].long()
        for x, y in ((K, cache.K), (V, cache.V)):
            x[:, :, :loop.N] = y[at, :, (rows % 16).expand_as(at)].transpose(1, 2)

    def prompt(n):
        lo = loop.N
        out = loop.prompt(*(x[:, lo:lo + n] for x in (q, k, v)))
        torch.cuda.synchronize()
        # the rotated queries once more, on their own
        lens = torch.full((B,), lo + n, dtype=torch.int32)
        cu = torch.arange(0, B * n + 1, n, dtype=torch.int32)
        q_rot, _, _, _ = ref.append(q[:, lo:lo + n].reshape(B * n, Hq, D).cpu(), k[:, lo:lo + n].reshape(B * n, Hkv, D).cpu(), v[:, lo:lo + n].reshape(B * n, Hkv, D).cpu(),
                                    cache.K.cpu(), cache.V.cpu(), c.table, cu, lens, Ncap, f.cpu(), False)
        q_rot = q_rot.to(dtype)
        want, _, mag = ref.attn(q_rot, cache.K.cpu(), cache.V.cpu(), c.table, cu, lens, Ncap, D ** -0.5)
        bound, _ = attn_bounds(c, q_rot, cache.K.cpu(), cache.V.cpu(), lo + n, D ** -0.5, mag, want)
        # (a query that the two round to different neighbours moves its scores by a step of its largest products)
        step = torch.finfo(dtype).eps * 1.01 if dtype != torch.float32 else 2.0 ** -20
        scores = step * D ** -0.5 * float(q_rot.double().norm(dim=-1).max() * torch.nan_to_num(cache.K.double()).norm(dim=-1).max())
        close(out.reshape(B * n, Hq, D), want, bound + 2 * scores * mag)

    t = 0

    def step():
        nonlocal flat, t
        n = loop.N
        out, lse = (x.clone() for x in loop.step(t, q[:, n], k[:, n], v[:, n], q_imp[n]))
        contiguous()
        if flat is None:
            flat = IntervalDecoder(K, V, W, Kimp, **kw)
        if t % P == 0:
            # every key is projected (sums of D products in fp32, rounded to the type), and the other loop gets the same ones: an fp32 sum depends on
            # how many rows are projected together
            keys, w = K[:, :, :n + 1].double().cpu(), W[0].double().cpu()
            want, mag = keys @ w, keys.abs() @ w.abs()
            close(loop.Kimp[:, :, :n + 1], want, mag * D * 2.0 ** -24 + (want.abs() * half_step(dtype) * 1.01 if dtype != torch.float32 else 0))
            assert not loop.Kimp[:, :, n + 1:].any()
            Kimp.copy_(loop.Kimp)
            flat.projected_upto = n + 1
        q_rot, k_rot = torch.empty_like(q[:, n]), torch.empty_like(k[:, n])
        tb.tb_append_paged_kv(tb.make_paged_desc(n + 1, Hq, cache), cache, q[:, n], k[:, n], v[:, n], None, loop.lens, f, q_rot, k_rot)
        o, l = flat.step(t, n + 1, q_rot, q_imp[n])
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, l)
        if t % P == 0:
            assert torch.equal(loop.idx, flat.idx) and torch.equal(loop.exp_cnt, flat.exp_cnt)
        t += 1

    prompt(100)
    prompt(57)
    for _ in range(8):
        step()
    prompt(31)  # rows that no prediction has seen, in the middle of an interval
    for _ in range(5):
        step()
    prompt(1)
    step()
    assert loop.N == 100 + 57 + 8 + 31 + 5 + 1 + 1
    with pytest.raises(ValueError):
        loop.prompt(*(x[:, :Ncap] for x in (q.repeat(1, 2, 1, 1), k.repeat(1, 2, 1, 1), v.repeat(1, 2, 1, 1))))
