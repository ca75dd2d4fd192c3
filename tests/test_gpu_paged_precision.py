"""How exact the calls on a cache in pages are, against 64 bits: weights of single tokens."""
import math

import pytest
import torch

from oracle import paged as ref
from paged_util import attn_bounds, close, half_step, make
from test_gpu_paged import BF, on_gpu, run_attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,new", [(4, 4, 1), (4, 2, 1), (8, 2, 1), (8, 1, 1), (4, 4, 5), (8, 4, 3), (8, 2, 2)])
@pytest.mark.parametrize("kept,window,holes", [([40, 0, 333, 3000], 0, ()), ([1700], 600, ()), ([90, 70], 0, [(0, 1), (1, 4)])])
def test_weights_of_up_to_eight_rows(D, Hq, Hkv, new, kept, window, holes):
    """bf16, weights close to each other and queries so small that scores are as good as exact: what is left are the weights, of which
    2^-16 may be lost at most (two roundings to bf16, of the weight and of what the first one left), and the result's rounding."""
    c = make(BF, Hq, Hkv, D, 16, [new] * len(kept), kept, seed=D + Hq + new, holes=holes)
    c.q = (c.q.float() * 0.05).to(BF)
    scale = D ** -0.5
    want, lse, mag = ref.attn(c.q, c.K, c.V, c.table, c.cu, c.lens, c.N, scale, window)
    on_gpu(c)
    out, l = run_attn(c, scale, window)
    tol, tol_lse = attn_bounds(c, c.q, c.K, c.V, c.N, scale, mag, want, exact_weights=True)
    close(out, want, tol + mag * half_step(BF) ** 2 * 1.01 + want.abs() * half_step(BF) * 1.01, "out")
    close(l, lse, tol_lse + lse.abs() * 2.0 ** -22, "lse")


@pytest.mark.parametrize("D", [64, 128])
def test_infinite_rows_that_all_see(D):
    """An infinite element among finite ones, behind a weight that 8 bits hold (1, of rows alike) or not: the infinity, not NaN."""
    c = make(BF, 4, 2, D, 16, [1, 2, 1], [200, 200, 37], seed=D)
    c.q[0] = 0
    for b, (n, value) in enumerate([(3, math.inf), (150, -math.inf), (37, math.inf)]):
        p, r = ref.place(c.table, b, n, 16, c.K.shape[0])
        c.V[p, :, r, 7] = value
    want, _, mag = ref.attn(c.q, c.K, c.V, c.table, c.cu, c.lens, c.N, D ** -0.5)
    assert bool(want[0, :, 7].isposinf().all()) and bool(want[1, :, 7].isneginf().all())
    on_gpu(c)
    out, _ = run_attn(c, D ** -0.5)
    tol, _ = attn_bounds(c, c.q, c.K, c.V, c.N, D ** -0.5, mag.nan_to_num(), want.nan_to_num(posinf=0, neginf=0), exact_weights=True)
    close(out, want, tol.nan_to_num(posinf=1e30) + mag.nan_to_num(posinf=0) * half_step(BF) ** 2 * 1.01 + want.nan_to_num(posinf=0, neginf=0).abs() * half_step(BF) * 1.01)
