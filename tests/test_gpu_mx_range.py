"""The 4-bit cache at the ends of what fp32 holds, and where the softmax's reference has to follow the scores through every grouping.

Logits rise along the rows by amounts that the reference of a running softmax may lag behind, so that it moves several times in every
wave with accumulators that hold something.  Bar: a logit is off by at most D roundings of its fp32 sum and four of the scale and the
exponential's argument, (D + 4) 2^-24 sum |q k| sm_scale; a weight by that share of itself, the mean of V by twice that of the largest
|V|; the sums of weights and rows by 1e-5 of it (160 roundings; a lane adds up at most 60 rows, and ten sums meet at the end)."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from oracle import mx
from paper_2503_07518_amd import binding as tb
from test_gpu_mx import BF16, F32, assert_attention, attend, coded_rows, mx_plan, mx_rows, randn, reference, say, score

pytestmark = pytest.mark.gpu

ROWS = 2800
RISE = 60.0  # from the first to the last row's logit, in powers of two


def rising(dtype, B, Hkv, g, D, byte, seed):
    """Rows whose logits rise for every head: element i of row n is the sign of the head's query there for i below D n / ROWS, its opposite
    from there on.  V: values above zero under one scale.  One cache for the whole batch; four different queries of it."""
    rng = np.random.default_rng(seed)
    sign = rng.choice([-1.0, 1.0], (Hkv, 1, D))
    z = np.abs(rng.standard_normal((4, Hkv, g, D))) + 0.2
    z *= RISE / 2 * np.log(2) / (z.sum(-1, keepdims=True) * D ** -0.5)
    q = torch.from_numpy((sign * z).reshape(4, Hkv * g, D)).to(dtype).repeat(B // 4, 1, 1).to(DEV)
    turned = np.arange(D)[None] < (np.arange(ROWS) * D / ROWS)[:, None]
    K, Kv = mx_rows((np.where(turned, 1.0, -1.0) * sign)[None])
    codes = torch.from_numpy(rng.integers(1, 8, (1, Hkv, ROWS, D // 2, 2)).astype(np.uint8))
    V = tb.MxRows((codes[..., 0] | codes[..., 1] << 4).to(DEV), torch.full((1, Hkv, ROWS, D // 32), byte, dtype=torch.uint8, device=DEV))
    Vv = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])[codes.numpy()].reshape(1, Hkv, ROWS, D) * 2.0 ** (byte - 127)

    def whole_batch(r):
        return tb.MxRows(r.codes.expand(B, -1, -1, -1), r.scales.expand(B, -1, -1, -1))

    return q, whole_batch(K), whole_batch(V), Kv, Vv


def check(dtype, D, g, kind, byte):
    B, Hkv = (64, 4) if kind != "lists" else (128, 4) if g == 1 else (64, 2)
    q, K, V, Kv, Vv = rising(dtype, B, Hkv, g, D, byte, 10 * g + D)
    heads = {"lists": Hkv * g, "shared": 1, "dense": 0}[kind]
    args = (None, None, 0, (0, ROWS))
    if heads:
        args = (torch.arange(ROWS, dtype=torch.int32, device=DEV).expand(B, heads, -1).contiguous(),
                torch.full((B, heads), ROWS, dtype=torch.int32, device=DEV), ROWS, (0, 0))
    by_group, splits = mx_plan(q, Hkv, ROWS, kind != "lists")
    assert by_group == (kind != "lists")
    step = splits * (256 if by_group else 128 * 128 // D)  # rows from a wave's tile to its next one
    assert RISE * step / ROWS < 8, "every step passes the reference's lag at once"
    out, lse = (t.cpu().numpy() for t in attend(q, K, V, ROWS, *args, shared=kind == "shared"))
    for b in range(4, B):
        assert np.array_equal(out[b], out[b % 4]) and np.array_equal(lse[b], lse[b % 4])
    Kv, Vv = (np.broadcast_to(x, (4,) + x.shape[1:]) for x in (Kv, Vv))
    few = args if not heads else (args[0][:4], args[1][:4], *args[2:])
    ref = reference(q[:4], Kv, Vv, ROWS, *few)
    assert np.exp(ref[1]).max() < 2.0 ** (RISE / 2 + 8), "the weights, of which the largest is 1, add up to less than 2^8"
    bar = 2 * (D + 4) * 2.0 ** -24 * (np.abs(q[:4].float().cpu().numpy()).sum(-1).max() * D ** -0.5) + 1e-5
    assert bool(np.isfinite(out).all())
    assert np.abs(out[:4] - ref[0]).max() <= bar * Vv.max()
    assert np.abs(lse[:4] - ref[1]).max() <= bar * np.abs(ref[1]).max()


KINDS = [("lists", 1), ("lists", 4), ("lists", 8), ("shared", 2), ("shared", 4), ("shared", 8), ("dense", 2), ("dense", 4), ("dense", 8)]


@pytest.mark.parametrize("kind,g", KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rising_logits_of_large_values(dtype, D, kind, g):
    """V of up to 6 * 2^117: times a sum of weights below 2^8, of which the largest is 1, less than 2^127.6.  With weights that are 2^4 times as
    large the sums would be infinite (some 80 rows count, the mean of V is 2.6 * 2^117)."""
    say(f"mx attention, rising logits, V near 2^120, {kind} {dtype} D={D} g={g}")
    check(dtype, D, g, kind, 244)


@pytest.mark.parametrize("kind,g", KINDS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_scale_and_large_products(dtype, kind, g):
    """sm_scale = 0 is the mean of the rows however large the products of queries and keys are (up to 2^126 here)."""
    say(f"mx attention, sm_scale=0, products near 2^126, {kind} {dtype} g={g}")
    B, Hkv, D, N = 13, 8, 128, 1200
    (K, Kv), (V, Vv) = coded_rows(1, Hkv, N, D, 1), coded_rows(1, Hkv, N, D, 2)
    K.scales.fill_(127 + 113)
    q = randn((B, Hkv * g, D), dtype, 3, 2.0 ** 6)
    codes = mx.dequantize(K.codes.cpu().numpy(), K.scales.cpu().numpy())[0]
    dots = np.abs(codes[:, None] @ q.float().cpu().numpy().reshape(B, Hkv, g, D).astype(np.float64).transpose(1, 0, 3, 2))
    assert 2.0 ** 125 < dots.max() < 2.0 ** 127
    whole = [tb.MxRows(r.codes.expand(B, -1, -1, -1), r.scales.expand(B, -1, -1, -1)) for r in (K, V)]
    heads = {"lists": Hkv * g, "shared": 1, "dense": 0}[kind]
    rows = N - 7
    args = (None, None, 0, (7, N))
    if heads:
        args = (torch.arange(7, N, dtype=torch.int32, device=DEV).expand(B, heads, -1).contiguous(),
                torch.full((B, heads), rows, dtype=torch.int32, device=DEV), rows, (0, 0))
    assert mx_plan(q, Hkv, rows, kind != "lists")[0] == (kind != "lists")
    for sm in (0.0, -0.0):
        got = attend(q, *whole, N, *args, sm=sm, shared=kind == "shared")
        mean = np.repeat(Vv[:, :, 7:].mean(2), g, 1)
        assert_attention(got, (np.broadcast_to(mean, (B, Hkv * g, D)), np.full((B, Hkv * g), np.log(rows))), Vv)


def strange_queries(dtype, B, Hkv, g, D, rows):
    """Queries, most of them ordinary, and rows in whose columns 3 and 40 there is no zero: column 3 has both signs, column 40 is below zero."""
    K, _ = coded_rows(B, Hkv, rows, D, 1)
    codes = K.codes
    codes[..., 1] = (codes[..., 1] & 0x0F) | 0x10 | (codes[..., 1] & 0xE0)   # element 3, the high half of byte 1: no zero
    codes[..., 20] = codes[..., 20] & 0xF0 | 0x09 | codes[..., 20] & 0x06     # element 40, the low half of byte 20: a sign, no zero
    q = randn((B, Hkv * g, D), dtype, 3, 0.5)
    heads = q.view(B, Hkv, g, D)
    heads[0, 0, 0, 3] = np.inf          # scores of both infinities: NaN
    heads[0, Hkv - 1, g - 1, 5] = np.nan
    heads[B - 1, 0, g - 1, 40] = np.inf   # minus infinity alone: as an empty list
    heads[B - 1, Hkv - 1, 0, 40] = -np.inf  # plus infinity alone: NaN
    return q, K, mx.dequantize(K.codes.cpu().numpy(), K.scales.cpu().numpy())


@pytest.mark.parametrize("kind,g", KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinite_and_nan_queries(dtype, D, kind, g):
    """What the formula makes of them, in their own head alone."""
    say(f"mx attention, infinite and NaN queries, {kind} {dtype} D={D} g={g}")
    B, Hkv, rows = 13, 8, 1200
    q, K, Kv = strange_queries(dtype, B, Hkv, g, D, rows)
    V, Vv = coded_rows(B, Hkv, rows, D, 2)
    heads = {"lists": Hkv * g, "shared": 1, "dense": 0}[kind]
    args = (None, None, 0, (0, rows))
    if heads:
        args = (torch.arange(rows, dtype=torch.int32, device=DEV).expand(B, heads, -1).contiguous(),
                torch.full((B, heads), rows, dtype=torch.int32, device=DEV), rows, (0, 0))
    assert mx_plan(q, Hkv, rows, kind != "lists")[0] == (kind != "lists")
    got = attend(q, K, V, rows, *args, shared=kind == "shared")
    with np.errstate(invalid="ignore"):
        ref = reference(q, Kv, Vv, rows, *args)
    empty = (B - 1, g - 1)
    assert np.isnan(ref[0][empty]).all()
    ref[0][empty], ref[1][empty] = 0.0, -np.inf
    strange = [(0, 0), (0, Hkv * g - 1), (B - 1, (Hkv - 1) * g)]
    assert np.isnan(ref[1]).sum() == len(set(strange)) and all(np.isnan(ref[0][at]).all() for at in strange)
    assert_attention(got, ref, Vv)


@pytest.mark.parametrize("g", [1, 2, 4, 8])
@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_of_infinite_and_nan_queries(dtype, d, g):
    say(f"mx score, infinite and NaN queries, {dtype} d'={d} g={g}")
    B, Hkv, N = 2, 2, 700
    K, Kv = coded_rows(B, Hkv, N, d, 1)
    q = randn((B, Hkv * g, d), dtype, 3)
    q[0, 0, 3], q[1, 0, 7], q[1, -1, 0] = np.inf, -np.inf, np.nan
    q[0, -1, 5] = 3e38 if dtype == F32 else 2.0 ** 127
    got = score(q, K, N).cpu().numpy()[..., :N]
    with np.errstate(invalid="ignore"):
        ref = np.einsum("bkgd,bknd->bkgn", q.float().cpu().numpy().astype(np.float64).reshape(B, Hkv, g, d), Kv).reshape(B, Hkv * g, N)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.isnan(ref).sum() > N and np.isinf(ref).sum() > N
    assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    fin = np.isfinite(ref) & (np.abs(ref) < 3.4e38)
    mag = np.einsum("bkgd,bknd->bkgn", np.abs(np.nan_to_num(q.float().cpu().numpy().astype(np.float64), posinf=0, neginf=0)).reshape(B, Hkv, g, d),
                    np.abs(Kv)).reshape(ref.shape)
    assert (np.abs(got[fin] - ref[fin]) <= (3 * d + 2) * 2.0 ** -24 * mag[fin]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_code_under_every_scale(dtype):
    """Bytes 253 and 254, which the library does not write, have codes beyond the largest number of either type: infinities."""
    say(f"mx, every code under every scale byte, {dtype}")
    codes = torch.arange(256, dtype=torch.uint8).view(16, 16).repeat(256, 1).reshape(1, 16, 256, 16).contiguous()
    scales = torch.arange(256, dtype=torch.uint8).repeat_interleave(16).reshape(1, 16, 256, 1).contiguous()
    rows = tb.MxRows(codes.repeat(1, 1, 1, 2).to(DEV), scales.repeat(1, 1, 1, 2).to(DEV))
    out = torch.zeros((1, 16, 256, 64), dtype=dtype, device=DEV)
    tb.tb_dequantize_mx(tb.make_desc(256, 16, K=out), rows, None, None, 0, out, None, None, 0, 256)
    got = out.float().cpu().numpy()
    with np.errstate(over="ignore"):
        want = mx.dequantize(rows.codes.cpu().numpy(), rows.scales.cpu().numpy()).astype(np.float32)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isinf(want).any(axis=-1).reshape(256, 16).any(1).nonzero()[0].tolist() == [253, 254]


@pytest.mark.parametrize("kind,g", KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_subnormal_rows_and_large_queries(dtype, D, kind, g):
    """Rows under the smallest scales, most of their elements subnormal numbers, and queries near the largest number: logits of a few units."""
    say(f"mx attention, subnormal rows, {kind} {dtype} D={D} g={g}")
    B, Hkv, rows = 13, 8, 1200
    (K, _), (V, Vv) = coded_rows(B, Hkv, rows, D, 1), coded_rows(B, Hkv, rows, D, 2)
    K.scales.copy_(K.scales % 3)
    Kv = mx.dequantize(K.codes.cpu().numpy(), K.scales.cpu().numpy())
    q = randn((B, Hkv * g, D), dtype, 3, 2.0 ** 123)
    heads = {"lists": Hkv * g, "shared": 1, "dense": 0}[kind]
    args = (None, None, 0, (0, rows))
    if heads:
        args = (torch.arange(rows, dtype=torch.int32, device=DEV).expand(B, heads, -1).contiguous(),
                torch.full((B, heads), rows, dtype=torch.int32, device=DEV), rows, (0, 0))
    assert mx_plan(q, Hkv, rows, kind != "lists")[0] == (kind != "lists")
    ref = reference(q, Kv, Vv, rows, *args)
    assert ref[1].max() > np.log(rows) + 0.1, "the rows make a difference"
    assert_attention(attend(q, K, V, rows, *args, shared=kind == "shared"), ref, Vv)
