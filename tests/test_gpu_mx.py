"""The cache in microscaled 4-bit floating point on the GPU: conversions bit for bit, scores and attention against the oracle in 64
bits on the values that the rows stand for.

Bars.  Codes, scales and converted rows: equal bits.  Scores: products are exact (an fp32 query is the sum of three bf16 numbers), so
only the fp32 sum rounds: at most 3 d' additions and the scale, (3 d' + 2) 2^-24 of sum |q k|.  Attention: 1e-5 of the largest |V| and
1e-5 of max(1, |lse|), the bar of fp32 rows (gpu_util.py): the queries' products are exact for both types here, and the softmax and its sums are
fp32, where an error of the logits of (D + 4) 2^-24 sum |q k| sm_scale, 8e-6 at D = 128 and a sum of one, moves a weight by that
share of itself and the mean of V by less."""
import ctypes
import math

import numpy as np
import pytest
import torch

from gpu_util import DEV, AttnPlan, gpu_select
from oracle import mx
from paper_2503_07518_amd import binding as tb
from paper_2503_07518_amd import interval
from test_gpu_offload import device_address

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def say(msg):
    print(f"[case] {msg}", flush=True)


def randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def mx_rows(x_np):
    """The oracle's codes of rows, on the GPU, and the values they stand for."""
    codes, scales = mx.quantize(x_np)
    return tb.MxRows(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV)), mx.dequantize(codes, scales)


def random_rows(B, Hkv, N, inner, seed):
    rng = np.random.default_rng(seed)
    return mx_rows(rng.standard_normal((B, Hkv, N, inner)) * np.exp(rng.standard_normal((1, Hkv, 1, inner)) / 2))


def coded_rows(B, Hkv, N, inner, seed):
    """Rows drawn as codes: every code as often, scales that differ."""
    rng = np.random.default_rng(seed)
    codes, scales = rng.integers(0, 256, (B, Hkv, N, inner // 2), dtype=np.uint8), rng.integers(122, 126, (B, Hkv, N, inner // 32), dtype=np.uint8)
    return tb.MxRows(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV)), mx.dequantize(codes, scales)


def side_by_side(K, V):
    """The same rows in a cache of the package's layout."""
    B, Hkv, N, half = K.codes.shape
    cache = tb.MxCache(B, Hkv, N, 2 * half, device=DEV)
    for to, frm in ((cache.K, K), (cache.V, V)):
        to.codes.copy_(frm.codes)
        to.scales.copy_(frm.scales)
    return cache.K, cache.V


# --------------------------------------------------------------------------- conversions

def special_rows(B, Hkv, n, inner, seed):
    """Rows of every size, with zeros, subnormals, halves between codes, infinities and NaN among them."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, Hkv, n, inner)) * np.exp2(rng.integers(-20, 20, (B, Hkv, n, 1)))
    blocks = x.reshape(-1, 32)
    for i, kind in enumerate(rng.integers(0, 12, len(blocks))):
        if kind == 0:
            blocks[i] = 0.0
        elif kind == 1:
            blocks[i] *= 2.0 ** -125
        elif kind == 2:
            blocks[i] = rng.choice([0, -0.0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, -2.5, -5], 32) * 2.0 ** rng.integers(-100, 100)
        elif kind == 3:
            blocks[i, rng.integers(32)] = rng.choice([np.inf, -np.inf, np.nan])
        elif kind == 4:
            blocks[i] *= 2.0 ** 100
    with np.errstate(over="ignore"):  # (what is too large for fp32 becomes an infinity there)
        return torch.from_numpy(x.astype(np.float32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hkv,n,D,Dimp", [(2, 3, 1, 128, 32), (16, 8, 1, 64, 64), (1, 2, 7, 64, 32), (3, 2, 1031, 128, 64), (1, 1, 4096, 128, 32),
                                            (2, 1, 129, 64, 32)])
def test_conversion_bits(dtype, B, Hkv, n, D, Dimp):
    say(f"mx conversion {dtype} B={B} Hkv={Hkv} rows={n} D={D} Dimp={Dimp}")
    x = [special_rows(B, Hkv, n, i, s).to(dtype).to(DEV) for s, i in enumerate((D, D, Dimp))]
    cache = tb.MxCache(B, Hkv, n, D, Dimp)
    q = (cache.K, cache.V, cache.Kimp)
    tb.tb_quantize_mx(tb.make_desc(n, Hkv, K=x[0], V=x[1], Kimp=x[2]), *x, 0, *q, 0, n)
    back = [torch.full_like(t, 7.0) for t in x]
    tb.tb_dequantize_mx(tb.make_desc(n, Hkv, K=back[0], V=back[1], Kimp=back[2]), *q, 0, *back, 0, n)
    torch.cuda.synchronize()
    for t, r, o in zip(x, q, back):
        codes, scales = mx.quantize(t.float().cpu().numpy().astype(np.float64))
        assert np.array_equal(r.scales.cpu().numpy(), scales)
        assert np.array_equal(r.codes.cpu().numpy(), codes)
        want = mx.dequantize(codes, scales).astype(np.float32)
        got = o.float().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("which", ["K", "V", "Kimp", "KV", "KKimp", "VKimp"])
def test_conversion_of_some_arrays_into_rows_of_a_larger_cache(dtype, which):
    say(f"mx conversion, {which} of three, row ranges, strides, {dtype}")
    B, Hkv, D, Dimp, n, src, dst, cap = 2, 2, 128, 32, 37, 5, 11, 64
    wide = [randn((Hkv, B, src + n + 3, i + 8), dtype, 5 + s).transpose(0, 1)[..., :i] for s, i in enumerate((D, D, Dimp))]
    taken = ["K" in which.replace("Kimp", ""), "V" in which, "Kimp" in which]
    rows, stores = [], []
    for i in (D, D, Dimp):  # an odd number of bytes between the scales of two rows, heads outermost
        codes = torch.full((Hkv, B, cap, i // 2 + 16), 0xA5, dtype=torch.uint8, device=DEV)
        scales = torch.full((Hkv, B, cap, i // 32 + 1), 0x5A, dtype=torch.uint8, device=DEV)
        stores += [(codes, 0xA5, i // 2), (scales, 0x5A, i // 32)]
        rows.append(tb.MxRows(codes.transpose(0, 1)[..., :i // 2], scales.transpose(0, 1)[..., :i // 32]))
    pick = lambda a: [t if on else None for t, on in zip(a, taken)]  # noqa: E731
    d = tb.make_desc(src + n + 1, Hkv, K=wide[0], V=wide[1], Kimp=wide[2])
    tb.tb_quantize_mx(d, *pick(wide), src, *pick(rows), dst, n)
    torch.cuda.synchronize()
    for t, on in enumerate(taken):
        if on:
            codes, scales = mx.quantize(wide[t][:, :, src:src + n].float().cpu().numpy())
            assert np.array_equal(rows[t].codes[:, :, dst:dst + n].cpu().numpy(), codes)
            assert np.array_equal(rows[t].scales[:, :, dst:dst + n].cpu().numpy(), scales)
        for store, fill, used in stores[2 * t:2 * t + 2]:  # nothing else is written
            keep = torch.ones(store.shape, dtype=torch.bool)
            if on:
                keep[:, :, dst:dst + n, :used] = False
            assert bool((store.cpu()[keep] == fill).all())
    out = [torch.full((B, Hkv, cap, i + 8), 7.0, dtype=dtype, device=DEV) for i in (D, D, Dimp)]
    view = [o[..., :i] for o, i in zip(out, (D, D, Dimp))]
    tb.tb_dequantize_mx(tb.make_desc(cap, Hkv, K=view[0], V=view[1], Kimp=view[2]), *pick(rows), dst, *pick(view), 3, n)
    torch.cuda.synchronize()
    for t, on in enumerate(taken):
        keep = torch.ones(out[t].shape, dtype=torch.bool)
        if on:
            got = view[t][:, :, 3:3 + n].float().cpu().numpy()
            assert np.array_equal(got, mx.dequantize(rows[t].codes[:, :, dst:dst + n].cpu().numpy(), rows[t].scales[:, :, dst:dst + n].cpu().numpy()))
            keep[:, :, 3:3 + n, :view[t].shape[3]] = False
        assert bool((out[t].cpu()[keep] == 7.0).all())


# --------------------------------------------------------------------------- scores

def score(q_imp, Kimp, N, scale=1.0, stride=None):
    B, Hq, _ = q_imp.shape
    scores = torch.full((B, Hq, stride or (N + 3) // 4 * 4), float("nan"), device=DEV)
    tb.tb_score_mx(tb.make_mx_desc(N, Hq, q_imp.dtype, Kimp=Kimp), q_imp, Kimp, scale, scores)
    torch.cuda.synchronize()
    return scores


def assert_score(got, q_imp, values, N, scale):
    B, Hq, d = q_imp.shape
    q = q_imp.float().cpu().numpy().astype(np.float64).reshape(B, values.shape[1], -1, d)
    k = values[:, :, :N]
    ref = scale * np.einsum("bkgd,bknd->bkgn", q, k).reshape(B, Hq, N)
    mag = abs(scale) * np.einsum("bkgd,bknd->bkgn", np.abs(q), np.abs(k)).reshape(B, Hq, N)
    err = np.abs(got[:, :, :N].cpu().numpy() - ref)
    assert (err <= (3 * d + 2) * 2.0 ** -24 * mag + 1e-38).all(), float((err / np.maximum(mag, 1e-30)).max())
    assert bool(torch.isnan(got[:, :, N:]).all()), "the padding of a row of scores is not written"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Dimp", [32, 64])
@pytest.mark.parametrize("B,Hkv,g,N", [(1, 1, 1, 1), (2, 3, 2, 5), (1, 2, 4, 256), (3, 1, 8, 257), (1, 8, 4, 4099), (2, 2, 1, 1023)])
def test_score(dtype, Dimp, B, Hkv, g, N):
    say(f"mx score {dtype} Dimp={Dimp} B={B} Hkv={Hkv} g={g} N={N}")
    rows, values = random_rows(B, Hkv, N + 3, Dimp, N)
    q_imp = randn((B, Hkv * g, Dimp), dtype, 3)
    for scale in (1.0, -0.37):
        assert_score(score(q_imp, rows, N, scale, (N + 11) // 4 * 4), q_imp, values, N, scale)


def test_score_of_strange_rows():
    """Strides of their own, and scales at both ends: products of subnormal rows and large queries are kept."""
    say("mx score, strides, extreme scales")
    B, Hkv, g, N, d = 2, 2, 4, 300, 32
    rng = np.random.default_rng(8)
    codes_np = rng.integers(0, 256, (B, Hkv, N, d // 2), dtype=np.uint8)
    scales_np = rng.choice([0, 1, 2, 3, 60, 127, 180], (B, Hkv, N, 1)).astype(np.uint8)
    scales_np[0, 1, 7] = 255
    codes = torch.zeros((Hkv, B, N, 48), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((B, N, Hkv, 3), dtype=torch.uint8, device=DEV)
    rows = tb.MxRows(codes.transpose(0, 1)[..., 16:32], scales.transpose(1, 2)[..., 1:2])
    rows.codes.copy_(torch.from_numpy(codes_np))
    rows.scales.copy_(torch.from_numpy(scales_np))
    q_imp = randn((B, Hkv * g, d), F32, 4, 2.0 ** 60)
    got = score(q_imp, rows, N)
    assert torch.isnan(got[0, g:, 7]).all() and int(torch.isnan(got).sum()) == g
    got[0, g:, 7] = 0
    values = mx.dequantize(codes_np, scales_np)
    values[0, 1, 7] = 0
    assert_score(got, q_imp, values, N, 1.0)


def test_scores_are_selected_from():
    """Quantise the projected keys, score, select: the scores' own top k."""
    say("mx project, quantise, score, select")
    B, Hkv, g, N, D, d, k = 1, 2, 4, 2000, 128, 32, 200
    K, W = randn((B, Hkv, N, D), BF16, 1), randn((1, D, d), BF16, 2, D ** -0.5)
    Kimp = torch.zeros((B, Hkv, N, d), dtype=BF16, device=DEV)
    desc = tb.make_desc(N, Hkv * g, K=K, Kimp=Kimp)
    tb.tb_project_keys(desc, K, W, Kimp, 0, N)
    cache = tb.MxCache(B, Hkv, N, D, d)
    tb.tb_quantize_mx(desc, None, None, Kimp, 0, None, None, cache.Kimp, 0, N)
    scores = score(randn((B, Hkv * g, d), BF16, 3), cache.Kimp, N)
    idx, cnt = gpu_select(scores, N, k, Hkv=Hkv)
    torch.cuda.synchronize()
    for h in range(Hkv * g):
        order = np.lexsort((np.arange(N), -scores[0, h].cpu().numpy().astype(np.float64)))
        assert np.array_equal(idx[0, h].cpu().numpy(), np.sort(order[:k]))


# --------------------------------------------------------------------------- attention

def attend(q, K, V, N, idx, cnt, max_count, tail=(0, 0), sm=None, ws=None, lse=True, stream=None, shared=None):
    B, Hq, D = q.shape
    shared = (idx is not None and idx.shape[1] != Hq) if shared is None else shared
    d = tb.make_mx_desc(N, Hq, q.dtype, K=K)
    ws = tb.new_workspace(tb.TB_OP_ATTN_MX, d, max_count + tail[1] - tail[0]) if ws is None else ws
    out = torch.full((B, Hq, D), float("nan"), device=DEV)
    l = torch.full((B, Hq), float("nan"), device=DEV) if lse else None
    call = tb.tb_sparse_decode_attn_shared_mx if shared else tb.tb_sparse_decode_attn_mx
    call(d, q, K, V, idx, cnt, max_count, D ** -0.5 if sm is None else sm, out, l, ws, *tail, stream=stream)
    return out, l


def reference(q, Kv, Vv, N, idx, cnt, max_count, tail=(0, 0), sm=None):
    """Row by row in 64 bits; entries outside the cache count as its first or last row, as for the other types."""
    q = q.float().cpu().numpy().astype(np.float64)
    B, Hq, D = q.shape
    g = Hq // Kv.shape[1]
    sm = D ** -0.5 if sm is None else sm
    out, lse = np.zeros((B, Hq, D)), np.full((B, Hq), -np.inf)
    for b in range(B):
        for h in range(Hq):
            rows = np.arange(*tail)
            if max_count:
                u = h if idx.shape[1] == Hq else 0
                n = min(max(int(cnt[b, u]), 0), max_count)
                rows = np.concatenate([np.clip(idx[b, u, :n].cpu().numpy(), 0, N - 1), rows]).astype(np.int64)
            if len(rows):
                x = sm * (Kv[b, h // g, rows] @ q[b, h])
                m = x.max()
                w = np.exp(x - m)
                lse[b, h] = m + np.log(w.sum())
                out[b, h] = (w / w.sum()) @ Vv[b, h // g, rows]
    return out, lse


def assert_attention(got, ref, Vv):
    out, lse = got[0].cpu().numpy().astype(np.float64), None if got[1] is None else got[1].cpu().numpy().astype(np.float64)
    bar = 1e-5 * max(1.0, float(np.nanmax(np.abs(Vv), initial=0.0)))
    assert np.array_equal(np.isnan(out), np.isnan(ref[0]))
    err = np.abs(np.nan_to_num(out) - np.nan_to_num(ref[0])).max(initial=0.0)
    assert err <= bar, f"max |out - oracle| = {err:.3e} > {bar:.3e}"
    if lse is not None:
        assert np.array_equal(np.isneginf(lse), np.isneginf(ref[1])) and np.array_equal(np.isnan(lse), np.isnan(ref[1]))
        fin = np.isfinite(ref[1])
        assert (np.abs(lse[fin] - ref[1][fin]) <= 1e-5 * np.maximum(1.0, np.abs(ref[1][fin]))).all()


def mx_plan(q, Hkv, rows, one_list):
    """Whether the library serves rows that all heads read by KV groups, and how many splits a head or group gets."""
    lib = tb.load_library()
    d = tb.tb_cache_desc(q.shape[0], q.shape[1], Hkv, q.shape[2], 32, tb.TB_F32 if q.dtype == F32 else tb.TB_BF16)
    grouped, by_head, by_group = (lib._ZN2tb15attn_mx_groupedEPK13tb_cache_descl, lib._ZN2tb12attn_mx_planEPK13tb_cache_descl,
                                  lib._ZN2tb18attn_mx_group_planEPK13tb_cache_descl)
    for f, kind in ((grouped, ctypes.c_bool), (by_head, AttnPlan), (by_group, AttnPlan)):
        f.restype, f.argtypes = kind, [ctypes.POINTER(tb.tb_cache_desc), ctypes.c_int64]
    by = one_list and grouped(ctypes.byref(d), rows)
    return by, (by_group if by else by_head)(ctypes.byref(d), rows).nsplit


def lists(B, heads, N, k, seed, ragged=True):
    """Ascending lists of up to k rows; ragged: an empty one, a single row, and lengths in between."""
    rng = np.random.default_rng(seed)
    idx, cnt = np.full((B, heads, max(k, 1)), -9, dtype=np.int32), np.zeros((B, heads), dtype=np.int32)
    for b in range(B):
        for h in range(heads):
            n = k
            if ragged:
                n = (0, 1, k, int(rng.integers(0, k + 1)))[(b * heads + h) % 4]
            idx[b, h, :n] = np.sort(rng.choice(N, n, replace=False))
            cnt[b, h] = n
    return torch.from_numpy(idx).to(DEV), torch.from_numpy(cnt).to(DEV)


CASES = [  # B, Hkv, g, N, k, tail rows
    (1, 1, 1, 1, 1, 0), (2, 2, 1, 40, 33, 0), (1, 2, 2, 300, 65, 7), (2, 1, 4, 700, 300, 1), (1, 8, 4, 3000, 700, 15), (1, 1, 8, 2000, 1900, 0),
    (3, 3, 2, 513, 129, 64), (9, 8, 1, 200, 31, 3), (8, 1, 2, 1500, 257, 0), (1, 1, 1, 9000, 8191, 5),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hkv,g,N,k,tail", CASES)
def test_attention_lists(dtype, D, B, Hkv, g, N, k, tail):
    say(f"mx attention {dtype} D={D} B={B} Hkv={Hkv} g={g} N={N} k={k} tail={tail}")
    (K, Kv), (V, Vv) = random_rows(B, Hkv, N, D, 1), random_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3)
    idx, cnt = lists(B, Hkv * g, N - tail, k, 4)
    t = (N - tail, N)
    got = attend(q, *side_by_side(K, V), N, idx, cnt, k, t)
    torch.cuda.synchronize()
    ref = reference(q, Kv, Vv, N, idx, cnt, k, t)
    assert_attention(got, ref, Vv)
    again = attend(q, K, V, N, idx, cnt, k, t)  # arrays of their own: the same sums
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hkv,g,N,k,tail", CASES)
def test_attention_shared_lists(dtype, D, B, Hkv, g, N, k, tail):
    say(f"mx attention, one list, {dtype} D={D} B={B} Hkv={Hkv} g={g} N={N} k={k} tail={tail}")
    (K, Kv), (V, Vv) = random_rows(B, Hkv, N, D, 1), random_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3)
    for ragged in (False, True):
        idx, cnt = lists(B, 1, N - tail, k, 4, ragged)
        t = (N - tail, N)
        got = attend(q, *side_by_side(K, V), N, idx, cnt, k, t, shared=True)
        torch.cuda.synchronize()
        assert_attention(got, reference(q, Kv, Vv, N, idx, cnt, k, t), Vv)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hkv,g,N,tail", [(1, 1, 1, 1, (0, 1)), (1, 1, 8, 1, (0, 1)), (2, 2, 4, 333, (0, 333)), (1, 2, 8, 5000, (17, 4999)),
                                            (3, 1, 2, 1000, (999, 1000)), (2, 8, 1, 2049, (0, 2049)), (1, 4, 4, 64, (5, 5)), (40, 8, 2, 70, (3, 70)),
                                            (4, 8, 4, 1111, (0, 1111)), (1, 1, 2, 20000, (0, 20000))])
@pytest.mark.parametrize("shared", [False, True])
def test_attention_dense(dtype, D, B, Hkv, g, N, tail, shared):
    say(f"mx attention, dense {dtype} D={D} B={B} Hkv={Hkv} g={g} rows {tail} of {N} shared={shared}")
    (K, Kv), (V, Vv) = random_rows(B, Hkv, N, D, 1), random_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3)
    got = attend(q, *side_by_side(K, V), N, None, None, 0, tail, shared=shared, lse=not shared)
    torch.cuda.synchronize()
    assert_attention(got, reference(q, Kv, Vv, N, None, None, 0, tail), Vv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,B,Hkv,g,N", [("lists", 3, 2, 4, 500), ("lists", 2, 8, 1, 700), ("shared", 13, 8, 8, 250), ("dense", 13, 8, 8, 251)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_strides(dtype, kind, B, Hkv, g, N, D):
    """One cache for the whole batch (a stride of 0), heads inside rows, scales at odd addresses with odd strides, K and V unlike."""
    say(f"mx attention, strides, {kind} {dtype} D={D} B={B} Hkv={Hkv} g={g} N={N}")
    (K1, Kv), (V1, Vv) = coded_rows(1, Hkv, N, D, 1), coded_rows(1, Hkv, N, D, 2)
    kc = torch.zeros((N, Hkv, D // 2 + 16), dtype=torch.uint8, device=DEV)
    ks = torch.full((N, Hkv, D // 32 + 1), 255, dtype=torch.uint8, device=DEV)
    vs = torch.full((Hkv, N, D // 32 + 2), 255, dtype=torch.uint8, device=DEV)
    kc[..., 16:].copy_(K1.codes[0].transpose(0, 1))
    ks[..., 1:].copy_(K1.scales[0].transpose(0, 1))
    vs[..., 1:-1].copy_(V1.scales[0])
    K = tb.MxRows(kc[..., 16:].transpose(0, 1)[None].expand(B, -1, -1, -1), ks[..., 1:].transpose(0, 1)[None].expand(B, -1, -1, -1))
    V = tb.MxRows(V1.codes.expand(B, -1, -1, -1), vs[..., 1:-1][None].expand(B, -1, -1, -1))
    Kv, Vv = (np.broadcast_to(x, (B,) + x.shape[1:]) for x in (Kv, Vv))
    q = randn((B, Hkv * g, D), dtype, 3)
    args = (None, None, 0, (1, N))
    if kind != "dense":
        k = N - 9 if kind == "shared" else 222
        idx, cnt = lists(B, 1 if kind == "shared" else Hkv * g, N, k, 4)
        args = (idx, cnt, k, (N - 9, N))
    assert mx_plan(q, Hkv, N, kind != "lists")[0] == (kind != "lists")
    got = attend(q, K, V, N, *args, shared=kind == "shared")
    torch.cuda.synchronize()
    assert_attention(got, reference(q, Kv, Vv, N, *args), Vv)


# one list or the dense range with enough heads and rows for a workgroup per KV group: B, Hkv, g, rows, splits
GROUPED = [(200, 8, 8, 16, 1), (850, 8, 2, 15, 1), (410, 8, 2, 31, 1), (60, 8, 4, 111, 1), (13, 8, 8, 250, 1), (6, 8, 8, 527, 2), (2, 4, 4, 6400, 25),
           (1, 8, 8, 3333, 13), (1, 2, 8, 38000, 68)]


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("B,Hkv,g,rows,splits", GROUPED)
@pytest.mark.parametrize("kind", ["dense", "shared"])
def test_attention_by_groups(dtype, D, B, Hkv, g, rows, splits, kind):
    say(f"mx attention by KV groups, {kind} {dtype} D={D} B={B} Hkv={Hkv} g={g} rows={rows}")
    N, tail = rows + 9, 3
    (K, Kv), (V, Vv) = coded_rows(B, Hkv, N, D, 1), coded_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3)
    if kind == "dense":
        args = (None, None, 0, (5, rows + 5))
    else:  # counts below the number that the call names, none at all among them
        idx, cnt = lists(B, 1, N - tail, rows - tail, 4)
        args = (idx, cnt, rows - tail, (N - tail, N))
    assert mx_plan(q, Hkv, rows, True) == (True, splits)
    got = attend(q, *side_by_side(K, V), N, *args, shared=True)
    torch.cuda.synchronize()
    ref = reference(q, Kv, Vv, N, *args)
    assert_attention(got, ref, Vv)
    again = attend(q, K, V, N, *args, shared=True)  # arrays of their own: the same sums
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("g,B,rows", [(8, 13, 250), (4, 4, 1700), (2, 20, 700)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["dense", "shared"])
def test_groups_of_strange_rows(dtype, D, g, B, rows, kind):
    """Rows that stand for NaN, attended to and not; entries outside the cache, counts below zero and beyond; scales of all signs."""
    say(f"mx attention by KV groups, strange rows, {kind} {dtype} D={D} g={g} B={B} rows={rows}")
    Hkv, N = 8, rows + 20
    (K, Kv), (V, Vv) = coded_rows(B, Hkv, N, D, 1), coded_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3, 0.5)

    def spoil(r, v, b, h, n, c):
        r.scales[b, h, n, c] = 255
        v[b, h, n, 32 * c:32 * c + 32] = np.nan

    spoil(K, Kv, 0, 0, 50, 1)
    spoil(V, Vv, 1, 1, 60, 0)
    for n in (0, 1, N - 1):  # attended to by nobody
        for c in range(D // 32):
            for r, v in ((K, Kv), (V, Vv)):
                r.scales[:, :, n, c] = 255
                v[:, :, n, 32 * c:32 * c + 32] = np.nan
    if kind == "dense":
        args = (None, None, 0, (2, rows + 2))
    else:
        rng = np.random.default_rng(3)
        idx = rng.integers(2, N - 1, (B, 1, rows + 7)).astype(np.int32)
        idx[:2, 0, :2] = (50, 60)
        idx[-1, 0, 3:7] = (-5, N, 2 ** 31 - 1, -2 ** 31)
        cnt = np.full((B, 1), rows - 13, dtype=np.int32)
        cnt[2], cnt[3] = -3, rows + 100
        args = (torch.from_numpy(idx).to(DEV), torch.from_numpy(cnt).to(DEV), rows, (2, 2))
    assert mx_plan(q, Hkv, rows, True)[0]
    with np.errstate(invalid="ignore"):
        for sm in (D ** -0.5, -0.1, 0.0):
            got = attend(q, *side_by_side(K, V), N, *args, sm=sm, shared=True)
            torch.cuda.synchronize()
            ref = reference(q, Kv, Vv, N, *args, sm=sm)
            assert 0 < np.isnan(ref[0]).sum() < ref[0].size
            assert_attention(got, ref, Vv)


@pytest.mark.parametrize("kind", ["dense", "shared"])
def test_groups_of_nan_rows_alone_and_of_growing_logits(kind):
    """Nothing but NaN; then logits that grow along the rows by far more than what a reference may lag behind, to several hundred."""
    say(f"mx attention by KV groups, NaN alone, growing logits, {kind}")
    B, Hkv, g, N, D = 2, 8, 8, 3000, 128
    rng = np.random.default_rng(5)
    q = randn((B, Hkv * g, D), BF16, 3, 4.0)
    qn = q.float().cpu().numpy().reshape(B, Hkv, g, D)[:, :, 0]
    x = rng.standard_normal((B, Hkv, N, D)) * 0.3 + np.sign(qn)[:, :, None] * np.linspace(-4, 4, N)[:, None]
    (K, Kv), (V, Vv) = mx_rows(x), coded_rows(B, Hkv, N, D, 2)
    idx = torch.arange(N, dtype=torch.int32, device=DEV).expand(B, 1, N).contiguous()
    args = (None, None, 0, (0, N)) if kind == "dense" else (idx, torch.full((B, 1), N, dtype=torch.int32, device=DEV), N, (0, 0))
    assert mx_plan(q, Hkv, N, True)[0]
    got = attend(q, K, V, N, *args, shared=True)
    torch.cuda.synchronize()
    ref = reference(q, Kv, Vv, N, *args)
    mag = (np.abs(q.float().cpu().numpy()).reshape(B, Hkv, g, D) @ np.abs(Kv).transpose(0, 1, 3, 2)).max() * D ** -0.5
    bar = 2 * (D + 4) * 2.0 ** -24 * mag  # what fp32 has of such logits, and of the weights
    assert mag > 100 and np.abs(got[0].cpu().numpy() - ref[0]).max() <= bar * np.abs(Vv).max() and np.abs(got[1].cpu().numpy() - ref[1]).max() <= bar
    K.scales.fill_(255)
    got = attend(q, K, V, N, *args, shared=True)
    assert torch.isnan(got[0]).all() and torch.isnan(got[1]).all()


@pytest.mark.parametrize("g,shared", [(1, False), (4, False), (4, True), (8, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_strange_lists(dtype, g, shared):
    """Counts below zero and above max_count, entries outside the cache, the same row twice, a list that ends the allocation."""
    say(f"mx attention, strange lists, {dtype} g={g} shared={shared}")
    B, Hkv, N, D, cap, most = 2, 2, 200, 64, 90, 77
    (K, Kv), (V, Vv) = random_rows(B, Hkv, N, D, 1), random_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3)
    heads = 1 if shared else Hkv * g
    rng = np.random.default_rng(3)
    idx = torch.from_numpy(rng.integers(0, N, (B, heads, cap)).astype(np.int32)).to(DEV)
    idx[0, 0, :4] = torch.tensor([-5, N, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64).to(torch.int32)
    cnt = torch.full((B, heads), 60, dtype=torch.int32, device=DEV)
    cnt[0, 0], cnt[-1, -1] = 1000, -3
    for tail in ((0, 0), (190, 200)):
        got = attend(q, K, V, N, idx, cnt, most, tail, shared=shared)
        torch.cuda.synchronize()
        assert_attention(got, reference(q, Kv, Vv, N, idx, cnt, most, tail), Vv)


@pytest.mark.parametrize("sm", [0.0, -0.11, 1e-30, 3.0])
@pytest.mark.parametrize("g,kind", [(4, "lists"), (2, "shared"), (8, "shared"), (4, "dense"), (1, "dense")])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_scales(dtype, g, kind, sm):
    """No scale at all (the mean of the rows), a negative one, and rows past the end in the last step."""
    say(f"mx attention, sm_scale={sm}, {dtype} g={g} {kind}")
    B, Hkv, N, D, k = 2, 2, 300, 64, 101
    (K, Kv), (V, Vv) = random_rows(B, Hkv, N, D, 1), random_rows(B, Hkv, N, D, 2)
    q = randn((B, Hkv * g, D), dtype, 3, 0.5)
    idx, cnt = lists(B, 1 if kind == "shared" else Hkv * g, N, k, 4, ragged=False)
    args = (None, None, 0, (0, N - 1)) if kind == "dense" else (idx, cnt, k, (0, 0))
    got = attend(q, K, V, N, *args, sm=sm, shared=kind == "shared")
    torch.cuda.synchronize()
    assert_attention(got, reference(q, Kv, Vv, N, *args, sm=sm), Vv)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,kind", [(1, "lists"), (4, "lists"), (2, "shared"), (4, "shared"), (8, "dense"), (1, "dense")])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_rows_that_stand_for_nan(dtype, D, g, kind):
    """NaN where an attended row makes it so, nowhere else: not from rows that nobody lists, nor from the slots past a list's end."""
    say(f"mx attention, NaN rows, {dtype} D={D} g={g} {kind}")
    B, Hkv, N, k = 2, 2, 400, 150
    (K, Kv), (V, Vv) = random_rows(B, Hkv, N, D, 1), random_rows(B, Hkv, N, D, 2)
    for r, v, at in ((K, Kv, (0, 0, 50, 1)), (V, Vv, (1, 1, 60, 0))):  # one block of one row each, attended to below
        r.scales[at] = 255
        v[at[:3]][32 * at[3]:32 * at[3] + 32] = np.nan
    for r, v in ((K, Kv), (V, Vv)):  # rows that no list names, the first among them
        for n in (0, 7, N - 1):
            r.scales[:, :, n] = 255
            v[:, :, n] = np.nan
    q = randn((B, Hkv * g, D), dtype, 3)
    heads = {"lists": Hkv * g, "shared": 1, "dense": 0}[kind]
    idx = cnt = None
    most, tail = 0, (8, N - 1)
    if heads:
        rng = np.random.default_rng(3)
        idx = np.stack([np.stack([np.sort(np.unique(np.concatenate([[50, 60], 8 + rng.permutation(N - 10)[:k]]))[:k]) for _ in range(heads)]) for _ in range(B)])
        idx, cnt = torch.from_numpy(idx.astype(np.int32)).to(DEV), torch.full((B, heads), k, dtype=torch.int32, device=DEV)
        most, tail = k, (9, 12)
        got = reference(q, Kv, Vv, N, idx, cnt, most, tail)[0]
    got = attend(q, *side_by_side(K, V), N, idx, cnt, most, tail, shared=kind == "shared")
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        ref = reference(q, Kv, Vv, N, idx, cnt, most, tail)
    assert 0 < np.isnan(ref[0]).sum() < ref[0].size
    assert_attention(got, ref, Vv)


@pytest.mark.parametrize("kind", ["lists", "shared", "dense"])
def test_attention_of_nan_rows_alone(kind):
    say(f"mx attention, nothing but NaN rows, {kind}")
    B, Hkv, g, N, D = 1, 2, 4, 3000, 128
    K, V = random_rows(B, Hkv, N, D, 1)[0], random_rows(B, Hkv, N, D, 2)[0]
    K.scales.fill_(255)
    q = randn((B, Hkv * g, D), BF16, 3)
    idx, cnt = lists(B, 1 if kind == "shared" else Hkv * g, N, 2900, 4, ragged=False)
    got = attend(q, K, V, N, None if kind == "dense" else idx, None if kind == "dense" else cnt, 0 if kind == "dense" else 2900,
                 (0, N) if kind == "dense" else (0, 0), shared=kind == "shared")
    torch.cuda.synchronize()
    assert torch.isnan(got[0]).all() and torch.isnan(got[1]).all()


@pytest.mark.parametrize("kind", ["lists", "shared", "dense"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_large_logits_and_one_dominant_row(dtype, kind):
    """Logits of hundreds: the running maximum has to keep up; the row that dominates is the answer."""
    say(f"mx attention, dominant row, {dtype} {kind}")
    B, Hkv, g, N, D = 1, 2, 4, 1500, 128
    rng = np.random.default_rng(5)
    x = rng.standard_normal((B, Hkv, N, D))
    q = randn((B, Hkv * g, D), dtype, 3, 20.0)
    x[:, :, 1400] = 4 * np.sign(q.float().cpu().numpy().reshape(B, Hkv, g, D)[:, :, 0])
    K, Kv = mx_rows(x)
    V, Vv = random_rows(B, Hkv, N, D, 2)
    heads = 1 if kind == "shared" else Hkv * g
    idx = torch.arange(N, dtype=torch.int32, device=DEV).expand(B, heads, N).contiguous()
    cnt = torch.full((B, heads), N, dtype=torch.int32, device=DEV)
    args = (None, None, 0, (0, N)) if kind == "dense" else (idx, cnt, N, (0, 0))
    got = attend(q, K, V, N, *args, shared=kind == "shared")
    torch.cuda.synchronize()
    ref = reference(q, Kv, Vv, N, *args)
    assert np.abs(ref[0][0, 0] - Vv[0, 0, 1400]).max() < 1e-6
    # logits of several hundred: fp32 has them to (D + 4) 2^-24 sum |q k| sm_scale, and a weight to that share
    mag = (np.abs(q.float().cpu().numpy()).reshape(B, Hkv, g, D) @ np.abs(Kv).transpose(0, 1, 3, 2)).max() * D ** -0.5
    bar = 2 * (D + 4) * 2.0 ** -24 * mag * np.abs(Vv).max()
    assert np.abs(got[0].cpu().numpy() - ref[0]).max() <= bar
    assert np.abs(got[1].cpu().numpy() - ref[1]).max() <= 2 * (D + 4) * 2.0 ** -24 * mag


def test_attention_row_offsets_past_31_bits():
    say("mx rows 4 GiB apart")
    B, Hkv, N, D, stride = 1, 1, (1 << 20) - 1, 128, 4096
    store = torch.zeros(N * stride, dtype=torch.uint8, device=DEV)
    codes = [store.as_strided((B, Hkv, N, D // 2), (N * stride, N * stride, stride, 1), 64 * t) for t in (0, 1)]
    scales = [store.as_strided((B, Hkv, N, D // 32), (N * stride, N * stride, stride, 1), 128 + 4 * t) for t in (0, 1)]
    K, V = (tb.MxRows(c, s) for c, s in zip(codes, scales))
    at = np.array([0, 1, 500000, 524287, 524288, 524289, 900001, N - 2, N - 1])
    x = [randn((B, Hkv, len(at), D), F32, 7 + t) for t in (0, 1)]
    for i, n in enumerate(at):  # the conversion reaches them, too
        tb.tb_quantize_mx(tb.make_desc(len(at), 1, K=x[0], V=x[1]), x[0], x[1], None, i, K, V, None, int(n), 1)
    small = [mx_rows(t.cpu().numpy()) for t in x]
    q = randn((1, 2, D), BF16, 3)
    idx = torch.from_numpy(at.astype(np.int32)).to(DEV).expand(1, 2, -1).contiguous()
    cnt = torch.full((1, 2), len(at), dtype=torch.int32, device=DEV)
    got = attend(q, K, V, N, idx, cnt, len(at))
    own = torch.arange(len(at), dtype=torch.int32, device=DEV).expand(1, 2, -1).contiguous()
    ref = reference(q, small[0][1], small[1][1], len(at), own, cnt, len(at))
    torch.cuda.synchronize()
    assert_attention(got, ref, small[1][1])
    got = attend(q, K, V, N, None, None, 0, (N - 2, N))
    torch.cuda.synchronize()
    assert_attention(got, reference(q, small[0][1], small[1][1], len(at), None, None, 0, (len(at) - 2, len(at))), small[1][1])


# --------------------------------------------------------------------------- workspaces, streams, graphs

def step(B, Hkv, g, N, D, k, dtype, seed):
    K, V = side_by_side(coded_rows(B, Hkv, N, D, seed)[0], coded_rows(B, Hkv, N, D, seed + 1)[0])
    idx, cnt = lists(B, Hkv * g, N, k, seed + 2, ragged=False)
    return dict(q=randn((B, Hkv * g, D), dtype, seed + 3), K=K, V=V, N=N, idx=idx, cnt=cnt, max_count=k)


def test_attention_repeats_bit_for_bit_and_leaves_the_workspace_ready():
    say("mx attention, 100 launches on one workspace, lists and dense in turn")
    s = step(1, 8, 4, 20000, 128, 3277, BF16, 1)
    dense = dict(q=s["q"], K=s["K"], V=s["V"], N=s["N"], idx=None, cnt=None, max_count=0, tail=(0, s["N"]))
    d = tb.make_mx_desc(s["N"], 32, BF16, K=s["K"])
    ws = tb.new_workspace(tb.TB_OP_ATTN_MX, d, s["N"])
    first = [attend(**x, ws=ws) for x in (s, dense)]
    for _ in range(50):
        for x, f in zip((s, dense), first):
            got = attend(**x, ws=ws)
            assert torch.equal(got[0], f[0]) and torch.equal(got[1], f[1])
    # room for fewer splits: another order of the sums, the same answer
    small = tb.new_workspace(tb.TB_OP_ATTN_MX, d, 1)
    with pytest.raises(tb.TbError) as e:
        attend(**dense, ws=small)
    assert e.value.code == tb.TB_ERR_WORKSPACE


def test_attention_on_another_stream():
    say("mx calls on another stream than the current one")
    s = step(2, 2, 4, 3000, 128, 500, BF16, 11)
    ref = attend(**s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    d = tb.make_mx_desc(s["N"], 8, BF16, K=s["K"])
    ws = tb.new_workspace(tb.TB_OP_ATTN_MX, d, 500)
    torch.cuda.synchronize()
    got = attend(**s, ws=ws, stream=side)
    side.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_attention_on_two_streams_at_once():
    """Calls that overlap, each on a workspace of its own; some by head, some by KV group."""
    say("mx attention on two streams at once")
    s = step(2, 8, 4, 6000, 128, 1500, BF16, 41)
    dense = dict(q=s["q"], K=s["K"], V=s["V"], N=s["N"], idx=None, cnt=None, max_count=0, tail=(0, s["N"]))
    ref = [attend(**x) for x in (s, dense)]
    d = tb.make_mx_desc(s["N"], 32, BF16, K=s["K"])
    ws = [tb.new_workspace(tb.TB_OP_ATTN_MX, d, s["N"]) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[(torch.empty_like(ref[0][0]), torch.empty_like(ref[0][1])) for _ in range(40)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(40):
        for w, st in enumerate(streams):
            x = (s, dense)[(i + w) % 2]
            tb.tb_sparse_decode_attn_mx(d, x["q"], x["K"], x["V"], x["idx"], x["cnt"], x["max_count"], 128 ** -0.5, *out[w][i], ws[w],
                                        *x.get("tail", (0, 0)), stream=st)
    torch.cuda.synchronize()
    for w in range(2):
        for i in range(40):
            want = ref[(i + w) % 2]
            assert torch.equal(out[w][i][0], want[0]) and torch.equal(out[w][i][1], want[1])


def test_two_graphs_share_a_workspace():
    """Two captured graphs on one workspace, replayed one after the other in either order."""
    say("mx attention, two graphs on one workspace")
    s = step(1, 8, 4, 6000, 128, 1500, BF16, 51)
    dense = dict(q=s["q"], K=s["K"], V=s["V"], idx=None, cnt=None, max_count=0, tail=(3, s["N"]))
    d = tb.make_mx_desc(s["N"], 32, BF16, K=s["K"])
    ws = tb.new_workspace(tb.TB_OP_ATTN_MX, d, s["N"])
    graphs, outs, refs = [], [], []
    side = torch.cuda.Stream()
    for x in (s, dense):
        o = (torch.zeros((1, 32, 128), device=DEV), torch.zeros((1, 32), device=DEV))

        def call():
            tb.tb_sparse_decode_attn_mx(d, x["q"], x["K"], x["V"], x["idx"], x["cnt"], x["max_count"], 0.09, *o, ws, *x.get("tail", (0, 0)))

        call()
        torch.cuda.synchronize()
        refs.append([t.clone() for t in o])
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                call()
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(g)
        outs.append(o)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1), (1, 0, 1)):
        for o in outs:
            for t in o:
                t.fill_(float("nan"))
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for o, r in zip(outs, refs):
            assert all(torch.equal(a, b) for a, b in zip(o, r)), order


def test_cache_in_host_memory():
    """Codes and scales in pinned host memory, as an offloaded cache has them: written, scored and attended to over the host link."""
    say("mx cache in pinned host memory")
    B, Hkv, g, N, D, d, k = 1, 2, 4, 900, 128, 32, 200
    x = [randn((B, Hkv, N, i), BF16, 60 + i) for i in (D, D + 2, d)]
    x[1] = x[1][..., :D].contiguous()
    src = tb.make_desc(N, Hkv * g, K=x[0], V=x[1], Kimp=x[2])
    q, q_imp = randn((B, Hkv * g, D), F32, 3), randn((B, Hkv * g, d), F32, 4)
    idx, cnt = lists(B, Hkv * g, N, k, 5)
    got = []
    for pinned in (False, True):
        def rows(inner):
            return tb.MxRows(*(torch.zeros((B, Hkv, N, n), dtype=torch.uint8, device="cpu" if pinned else DEV, pin_memory=pinned)
                               for n in (inner // 2, inner // 32)))
        K, V, Kimp = rows(D), rows(D), rows(d)
        if pinned and any(device_address(t) != t.data_ptr() for r in (K, V, Kimp) for t in (r.codes, r.scales)):
            pytest.skip("pinned host memory is not mapped at the same address for the device on this box")
        tb.tb_quantize_mx(src, *x, 0, K, V, Kimp, 0, N)
        got.append((score(q_imp, Kimp, N), *attend(q, K, V, N, idx, cnt, k), *attend(q, K, V, N, None, None, 0, (0, N))))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["lists", "shared", "dense"])
def test_steps_in_a_graph(kind):
    """Append, score and attention captured together; replays with new rows and other lists, eager work in between."""
    say(f"mx step under capture, {kind}")
    B, Hkv, g, N, D, d, k = 2, 2, 4, 3000, 128, 32, 700
    s = step(B, Hkv, g, N, D, k, BF16, 21)
    Kimp = random_rows(B, Hkv, N, d, 5)[0]
    K, V, q, q_imp = s["K"], s["V"], s["q"], randn((B, Hkv * g, d), BF16, 6)
    new = [randn((B, Hkv, 1, i), BF16, 30 + i) for i in (D, D + 1, d)]
    new[1] = new[1][..., :D].contiguous()
    src = tb.make_desc(1, Hkv * g, K=new[0], V=new[1], Kimp=new[2])
    desc = tb.make_mx_desc(N, Hkv * g, BF16, K=K, Kimp=Kimp)
    ws = tb.new_workspace(tb.TB_OP_ATTN_MX, desc, k + N)
    scores = torch.zeros((B, Hkv * g, N), device=DEV)
    out, lse = torch.zeros((B, Hkv * g, D), device=DEV), torch.zeros((B, Hkv * g), device=DEV)
    idx, cnt = (s["idx"], s["cnt"]) if kind == "lists" else lists(B, 1, N, k, 9, ragged=False)

    def run():
        tb.tb_quantize_mx(src, *new, 0, K, V, Kimp, N - 1, 1)
        tb.tb_score_mx(desc, q_imp, Kimp, 1.0, scores)
        if kind == "lists":
            tb.tb_sparse_decode_attn_mx(desc, q, K, V, idx, cnt, k, D ** -0.5, out, lse, ws, N - 1, N)
        elif kind == "shared":
            tb.tb_sparse_decode_attn_shared_mx(desc, q, K, V, idx, cnt, k, D ** -0.5, out, lse, ws, N - 1, N)
        else:
            tb.tb_sparse_decode_attn_mx(desc, q, K, V, None, None, 0, D ** -0.5, out, lse, ws, 0, N)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.current_stream().wait_stream(side)
    for r in range(4):
        for t in new:
            t.copy_(randn(t.shape, BF16, 100 + r))
        q.copy_(randn(q.shape, BF16, 200 + r))
        idx.copy_(lists(B, idx.shape[1], N, k, 300 + r, ragged=False)[0])
        run()  # eager, on the same workspace
        torch.cuda.synchronize()
        want = [t.clone() for t in (scores, out, lse, K.codes, V.scales)]
        for t in (scores, out, lse):
            t.fill_(float("nan"))
        K.codes[:, :, N - 1] = 0
        V.scales[:, :, N - 1] = 0
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((scores, out, lse, K.codes, V.scales), want):
            assert torch.equal(got, ref), f"replay {r}"


# --------------------------------------------------------------------------- the interval loop

@pytest.mark.parametrize("dtype,headless,mode,expand", [(BF16, False, 0, False), (F32, False, 1, True), (BF16, True, 0, False)])
def test_interval_loop(oracle, monkeypatch, dtype, headless, mode, expand):
    """A prompt, then single rows and steps; every stage against the oracle on what the stage before has left on the GPU."""
    say(f"mx interval loop {dtype} headless={headless} mode={mode} expand_on_predict={expand}")
    B, Hkv, g, D, d, N0, k, P, radius, sink, window = 2, 2, 4, 128, 32, 700, 60, 4, 1, 5, 9
    Hq, Ncap, dn = Hkv * g, N0 + 30, "f32" if dtype == F32 else "bf16"
    K, V = randn((B, Hkv, Ncap, D), dtype, 1), randn((B, Hkv, Ncap, D), dtype, 2)
    W = randn((1, D, d), dtype, 3, D ** -0.5)
    cache = tb.MxCache(B, Hkv, Ncap, D, 0 if headless else d)
    if headless:
        one = randn((B, 1, Ncap, d), dtype, 4)
        cache.Kimp = tb.MxCache(B, 1, Ncap, D, d).Kimp
        tb.tb_quantize_mx(tb.make_desc(Ncap, 1, Kimp=one), None, None, one, 0, None, None, cache.Kimp, 0, Ncap)
    monkeypatch.setattr(interval.MxIntervalDecoder, "PROJECT_ROWS", 256)  # the prompt in three pieces
    loop = interval.MxIntervalDecoder(cache, None if headless else W, Hq, k, P, radius, sink=sink, window=window, sm_scale=D ** -0.5, mode=mode,
                                      expand_on_predict=expand, headless=headless, dtype=dtype)
    loop.append(K[:, :, :N0 - 3], V[:, :, :N0 - 3])
    loop.append(K[:, :, N0 - 3:N0], V[:, :, N0 - 3:N0])
    kept = None
    for t in range(11):
        N = N0 + t
        if t:
            loop.append(K[:, :, N - 1:N], V[:, :, N - 1:N])
        assert loop.N == N
        q, q_imp = randn((B, Hq, D), dtype, 100 + t), randn((B, 1 if headless else Hq, d), dtype, 200 + t)
        out, lse = loop.step(t, q, q_imp)
        torch.cuda.synchronize()
        for rows, x in ((cache.K, K), (cache.V, V)):
            codes, scales = mx.quantize(x[:, :, :N].float().cpu().numpy())
            assert np.array_equal(rows.codes[:, :, :N].cpu().numpy(), codes) and np.array_equal(rows.scales[:, :, :N].cpu().numpy(), scales)
        Kv, Vv, Iv = (mx.dequantize(r.codes.cpu().numpy(), r.scales.cpu().numpy()) for r in (cache.K, cache.V, cache.Kimp))
        if t % P == 0:
            if not headless:  # the projected keys are those of the rows in their own type
                Kimp = torch.zeros((B, Hkv, N, d), dtype=dtype, device=DEV)
                tb.tb_project_keys(tb.make_desc(N, Hkv, K=K, Kimp=Kimp), K, W, Kimp, 0, N)
                near = mx.dequantize(*mx.quantize(Kimp.float().cpu().numpy()))
                # (another number of rows a call may sum in another order: the values themselves are near, a code next to a border moves)
                assert np.mean(near == Iv[:, :, :N]) > 0.999
                assert np.abs(near - Iv[:, :, :N]).max() <= 0.5 * np.abs(near).max()
            scores = loop.scores[:, :, :N]
            assert_score(torch.nn.functional.pad(scores, (0, 1), value=float("nan")), q_imp, Iv, N, 1.0)
            idx, cnt = oracle.select_topk(scores.cpu().numpy(), k, sink, window)
            assert np.array_equal(loop.cnt.cpu().numpy(), cnt) and np.array_equal(loop.idx.cpu().numpy()[:, :, :idx.shape[2]], idx)
            exp = oracle.expand_neighbors(idx, cnt, N, radius, mode=mode)
            for b in range(B):
                for h in range(idx.shape[1]):
                    n = int(exp[1][b, h])
                    assert int(loop.exp_cnt[b, h]) == n and np.array_equal(loop.exp_idx[b, h, :n].cpu().numpy(), exp[0][b, h, :n])
            kept = N
        if t % P == 0 and not expand:
            ref = reference(q, Kv, Vv, N, loop.idx, loop.cnt, loop.sel_cap)
        else:
            ref = reference(q, Kv, Vv, N, loop.exp_idx, loop.exp_cnt, loop.exp_cap, (kept, N))
        assert_attention((out, lse), ref, Vv)
    with pytest.raises(ValueError):
        loop.append(K, V)


@pytest.mark.parametrize("headless", [False, True])
def test_interval_loop_many_rows_between_predictions(headless):
    """More rows than P, and none at all, between two predictions: a conversation goes on with a prompt."""
    say(f"mx interval loop, many rows between predictions, headless={headless}")
    B, Hkv, g, D, d, N0, N1, k, P, radius = 1, 2, 2, 64, 32, 300, 5000, 40, 4, 1
    Hq = Hkv * g
    K, V = randn((B, Hkv, N1, D), BF16, 1), randn((B, Hkv, N1, D), BF16, 2)
    cache = tb.MxCache(B, Hkv, N1, D, 0 if headless else d)
    if headless:
        one = randn((B, 1, N1, d), BF16, 4)
        cache.Kimp = tb.MxCache(B, 1, N1, D, d).Kimp
        tb.tb_quantize_mx(tb.make_desc(N1, 1, Kimp=one), None, None, one, 0, None, None, cache.Kimp, 0, N1)
    loop = interval.MxIntervalDecoder(cache, None if headless else randn((1, D, d), BF16, 3, D ** -0.5), Hq, k, P, radius, sm_scale=D ** -0.5,
                                      headless=headless)
    Kv, Vv = (mx.dequantize(*mx.quantize(x.float().cpu().numpy())) for x in (K, V))
    have = 0
    for t, N in enumerate((N0, N0 + 1, N0 + 1, N1, N1)):
        loop.append(K[:, :, have:N], V[:, :, have:N])
        have = N
        q, q_imp = randn((B, Hq, D), BF16, 100 + t), randn((B, 1 if headless else Hq, d), BF16, 200 + t)
        got = loop.step(t, q, q_imp)
        torch.cuda.synchronize()
        assert loop.N == N
        args = (loop.idx, loop.cnt, loop.sel_cap) if t % P == 0 else (loop.exp_idx, loop.exp_cnt, loop.exp_cap, (N0, N))
        assert_attention(got, reference(q, Kv, Vv, N, *args), Vv)
