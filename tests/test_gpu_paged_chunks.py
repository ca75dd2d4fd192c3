"""Attention of chunks over pages in the shapes that only long calls take, against 64 bits on the GPU: eight waves a workgroup, and rows that
workgroups share; with windows, holes, infinite and NaN rows, ragged batches and tokens that take no part."""
import math

import pytest
import torch

from oracle import paged as ref
from paged_util import attn_bounds, close, make
from test_gpu_paged import BF, DEV, F32, check_attn, on_gpu, run_attn

pytestmark = pytest.mark.gpu


def eight_waves(c):
    """The rule by which eight waves of 32 rows share a tile of keys."""
    rows = c.T * c.Hq
    return c.dtype == BF and c.D == 128 and rows >= (64 if c.B == 1 else 256) * 256 and (rows >= 512 * 256 or c.N >= 4 * c.T)


def exact(c, b, h, window, scale, max_new):
    """Numbers of sequence b's tokens that take part, and of query head h their outputs, log-sum-exps and mean |V|, in 64 bits."""
    n, first = int(c.lens[b]), int(c.cu[b])
    new = int(c.cu[b + 1]) - first
    i = torch.arange(min(new, max_new))
    p = n - new + i
    i, p = i[(p >= 0) & (p < c.N)], p[(p >= 0) & (p < c.N)].to(DEV)[:, None]
    rows = torch.arange(min(n, c.N))
    page = c.table[b, rows // c.page].long()
    rows = rows[(page >= 0) & (page < c.K.shape[0])]
    at, hkv = c.table[b, rows // c.page].long(), h * c.Hkv // c.Hq
    K, V = (x[at, hkv, rows % c.page].to(DEV).double() for x in (c.K, c.V))
    rows = rows.to(DEV)
    seen = (rows <= p) & ((rows > p - window) if window else True)
    x = (c.q[first + i, h].to(DEV).double() @ K.T * scale).masked_fill_(~seen, -math.inf)
    lse = torch.logsumexp(x, 1)
    w = torch.exp(x - lse.nan_to_num(neginf=0)[:, None]).masked_fill_(~seen, 0)  # (nothing seen: all of them 0)
    finite = torch.where(V.isfinite(), V, 0)
    out, mag = w @ finite, w @ finite.abs()
    for r in (~V.isfinite()).any(1).nonzero().flatten().tolist():
        sees = seen[:, r]
        out[sees] += w[sees, r, None] * torch.where(V[r].isfinite(), 0, V[r])
    return first + i, out, lse, mag


def check(c, window=0, max_new=None, cu=True, heads=None):
    scale = c.D ** -0.5
    on_gpu(c)
    out, lse = (x.cpu() for x in run_attn(c, scale, window, max_new, cu))
    took = []
    for b in range(c.B):
        for h in range(c.Hq) if heads is None else heads:
            t, want, l, mag = (x.cpu() for x in exact(c, b, h, window, scale, c.most if max_new is None else max_new))
            tol, tol_lse = attn_bounds(c, c.q, c.K, c.V, c.N, scale, mag.nan_to_num(), want.nan_to_num(posinf=0, neginf=0))
            close(out[t, h], want, tol, f"out, sequence {b}, head {h}")
            close(lse[t, h], l, tol_lse + l.abs().nan_to_num(posinf=0) * 2.0 ** -22, f"lse, sequence {b}, head {h}")
        took += t.tolist()
    rest = [t for t in range(c.T) if t not in set(took)]
    assert bool((out[rest] == 7).all()) and bool((lse[rest] == 7).all())
    return out, lse


def spoil(c, b, window, back=((0, "V", math.inf), (3, "K", math.nan), (70, "V", -math.inf), (130, "V", math.nan))):
    """Infinite and NaN elements of sequence b's newest rows, and of one at the edge of its first tokens' window."""
    n, new = int(c.lens[b]), int(c.cu[b + 1] - c.cu[b])
    places = [(n - 1 - k, what, value) for k, what, value in back if k < new]
    if window:
        places.append((n - new - window + 5, "V", math.inf))
    for j, (row, what, value) in enumerate(places):
        at = ref.place(c.table, b, row, c.page, c.K.shape[0]) if row >= 0 else None
        if at:
            getattr(c, what)[at[0], j % c.Hkv, at[1], 9 + 40 * (j % 2)] = value


# ---- eight waves ------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hq", [64, 8])
@pytest.mark.parametrize("window", [0, 1, 200, 1000])
@pytest.mark.parametrize("page", [16, 64])
def test_windows(Hq, window, page):
    new = 300 * 64 // Hq
    c = make(BF, Hq, 8, 128, page, [new], [3 * new + 11], seed=window)
    assert eight_waves(c)
    check(c, window, heads=range(0, Hq, 3))


@pytest.mark.parametrize("Hq,Hkv", [(64, 8), (32, 8), (32, 16), (16, 16)])
@pytest.mark.parametrize("window", [0, 333])
def test_holes(Hq, Hkv, window):
    """Holes in front, in the middle of what is seen, and among the new rows; some tokens with a window see nothing else."""
    new = 300 * 64 // Hq
    c = make(BF, Hq, Hkv, 128, 16, [new], [3 * new + 1], seed=Hq, holes=[(0, 0), (0, 3), *((0, 30 + i) for i in range(25)), (0, (3 * new) // 16 + 2), (0, (4 * new) // 16 - 1)])
    assert eight_waves(c)
    check(c, window, heads=range(0, Hq, 3))


def test_tokens_that_see_holes_alone():
    c = make(BF, 64, 8, 128, 16, [300], [1000], seed=5, holes=[(0, i) for i in range(64, 70)])
    assert eight_waves(c)
    out, lse = check(c, window=20, heads=range(0, 64, 5))
    assert bool((lse[70:100] == -math.inf).all()) and not bool(out[70:100].any())


@pytest.mark.parametrize("Hq,Hkv", [(64, 8), (16, 8)])
@pytest.mark.parametrize("window", [0, 200])
def test_infinite_rows(Hq, Hkv, window):
    new = 300 * 64 // Hq
    c = make(BF, Hq, Hkv, 128, 16, [new], [3 * new + 11], seed=window)
    spoil(c, 0, window)
    assert eight_waves(c)
    check(c, window)


@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("spoilt", [False, True])
def test_ragged_batches(window, spoilt):
    """A token, chunks and a sequence without new tokens in one call, with holes; then with infinite rows."""
    c = make(BF, 64, 8, 128, 16, [1, 700, 0, 400, 2], [3000, 100, 20, 4600, 77], seed=6, holes=[(0, 9), (1, 2), (1, 40), (3, 100), (4, 1)], pad=3)
    assert eight_waves(c)
    if spoilt:
        for b in (0, 1, 3, 4):
            spoil(c, b, window)
    check(c, window, heads=range(0, 64, 7))


def test_tokens_without_a_place():
    """Fewer rows than tokens, rows past the last one, more tokens than the call says."""
    c = make(BF, 64, 8, 128, 16, [524, 300, 200], [0, 4000, 900], seed=7, pad=2)
    c.lens[0] = 450
    c.N = 4280
    assert eight_waves(c)
    check(c, heads=range(0, 64, 9))
    check(c, max_new=250, heads=range(0, 64, 9))


@pytest.mark.parametrize("window", [0, 900])
def test_a_prompt(window):
    """Rows enough for eight waves whatever the cache holds, as many tokens for each of two sequences, without cu."""
    c = make(BF, 32, 8, 128, 64, [2100, 2100], [0, 0], seed=8, holes=[(0, 3), (1, 20)])
    spoil(c, 1, window)
    assert eight_waves(c)
    check(c, window, cu=False, heads=range(0, 32, 7))


# ---- rows that workgroups share ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 2500])
@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (4, 4)])
def test_split_rows_with_holes(dtype, D, window, Hq, Hkv):
    """Splits of 1024 rows and up (fp32: 128 or 256), some of them with holes alone."""
    holes = [(0, e) for e in (*range(10, 90), 120, 200, 262)] + [(1, e) for e in (0, 3, *range(100, 130))]
    c = make(dtype, Hq, Hkv, D, 16, [33, 20], [4200, 2100], seed=D, holes=holes)
    check(c, window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 2500])
def test_split_rows_with_infinite_rows(dtype, D, window):
    c = make(dtype, 4, 2, D, 16, [150], [4200], seed=D + 1, holes=[(0, 260)])
    spoil(c, 0, window)
    check(c, window)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_split_rows_of_which_a_split_is_not_a_number(dtype):
    """NaN and infinite rows that all tokens see, in the first split alone: the sum of the splits has them."""
    c = make(dtype, 4, 2, 64, 16, [40], [4200], seed=9)
    for row, what, h, value in ((5, "K", 0, math.nan), (17, "V", 1, math.inf), (4100, "V", 1, -math.inf)):
        p, r = ref.place(c.table, 0, row, 16, c.K.shape[0])
        getattr(c, what)[p, h, r, 3] = value
    out, lse = check(c)
    assert bool(out[:, :2].isnan().all()) and bool(lse[:, :2].isnan().all()) and bool(lse[:, 2:].isfinite().all())
