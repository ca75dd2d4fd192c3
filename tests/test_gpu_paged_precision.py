"""How exact the calls on a cache in pages are, against 64 bits: weights of single tokens, rotated rows."""
import math

import pytest
import torch

from oracle import paged as ref
from paper_2503_07518_amd import binding as tb
from paged_util import attn_bounds, close, half_step, make
from test_gpu_paged import BF, DEV, F32, inv_freq, on_gpu, run_attn

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


# ---- rotation -----------------------------------------------------------------------------------------
def rotated(c, f, interleaved, positions=None):
    """Rotated queries and keys, and the keys in the cache, as the call leaves them."""
    on_gpu(c)
    qo, ko = torch.zeros(c.q.shape, dtype=c.dtype, device=DEV), torch.zeros(c.k.shape, dtype=c.dtype, device=DEV)
    tb.tb_append_paged_kv(c.desc, c.cache, c.q.to(DEV), c.k.to(DEV), c.v.to(DEV), c.cu.to(DEV), c.lens.to(DEV), f.to(DEV), qo, ko,
                          positions=None if positions is None else positions.to(DEV), interleaved=interleaved)
    torch.cuda.synchronize()
    return qo, ko


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,rot", [(4, 2, 64, 64), (4, 1, 128, 128), (32, 8, 128, 128), (16, 4, 64, 32), (2, 1, 128, 48)])
def test_fp32_rows_are_rounded_once(Hq, Hkv, D, rot, interleaved):
    """Positions below 2^17, where 64 bits leave 2^17 2^-53 of an angle uncertain, in the call's as in the reference's; what is computed in 64 bits
    from there adds less than 2^-40.  The rest is one rounding: half a step of the result."""
    c = make(F32, Hq, Hkv, D, 16, [40, 1, 3], [0, 333, 0], seed=rot)
    positions = torch.randint(0, 1 << 17, (c.T,), generator=c.gen, dtype=torch.int32)
    f = inv_freq(rot)
    for at in (None, positions):
        q, k, _, _ = ref.append(c.q, c.k, c.v, c.K, c.V, c.table, c.cu, c.lens, c.N, f, interleaved, at)
        for got, x, want in zip(rotated(c, f, interleaved, at), (c.q, c.k), (q, k)):
            close(got, want, want.abs() * half_step(F32) + x.double().abs().amax(-1, keepdim=True) * 2 * 2.0 ** -35)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("most", [1.0, 1000.0])
def test_far_positions(most, interleaved):
    """Angles of up to 2^41: a turn's part is as exact as at position 1."""
    c = make(F32, 4, 1, 128, 16, [8, 3], [1, 2], seed=11)
    positions = torch.tensor([2 ** 31 - 1, -2 ** 31, 999999937, -5, 1 << 30, 131071, 1 << 24, 1234567891, 1, 0, 2 ** 31 - 2], dtype=torch.int32)
    f = inv_freq(128) * most
    f[1::7] *= -1
    q, k, _, _ = ref.append(c.q, c.k, c.v, c.K, c.V, c.table, c.cu, c.lens, c.N, f, interleaved, positions)
    for got, x, want in zip(rotated(c, f, interleaved, positions), (c.q, c.k), (q, k)):
        close(got, want, want.abs() * half_step(F32) + x.double().abs().amax(-1, keepdim=True) * 2 * 2.0 ** -40)
