"""Caches in pages for the tests, on the CPU: everything that no sequence owns is NaN, so that whatever reads it is seen."""
from __future__ import annotations

import math
import types

import torch

U = 2.0 ** -24  # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def make(dtype, Hq, Hkv, D, page, new, kept, seed=0, spare=2, holes=(), pad=0):
    """new, kept: tokens and rows before them of every sequence; holes: (sequence, entry) of the table; pad: tokens behind the last one's."""
    gen = torch.Generator().manual_seed(seed)
    lens = [n + k for n, k in zip(new, kept)]
    B, T = len(new), sum(new) + pad
    entries = max(1, max(-(-max(n, 1) // page) for n in lens))
    pages = B * entries + spare
    c = types.SimpleNamespace(dtype=dtype, Hq=Hq, Hkv=Hkv, D=D, page=page, B=B, T=T, N=max(1, max(lens)), most=max(new + [1]))
    c.table = torch.randperm(pages, generator=gen)[:B * entries].view(B, entries).to(torch.int32)
    c.lens = torch.tensor(lens, dtype=torch.int32)
    c.cu = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32)
    c.K, c.V = (torch.full((pages, Hkv, page, D), math.nan, dtype=dtype) for _ in range(2))
    for b, n in enumerate(lens):
        for r in range(max(n, 0)):
            p = int(c.table[b, r // page])
            for x in (c.K, c.V):
                x[p, :, r % page] = torch.randn((Hkv, D), generator=gen).to(dtype)
    for i, (b, e) in enumerate(holes):
        c.table[b, e] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[i % 4]
    c.q = (1.5 * torch.randn((T, Hq, D), generator=gen)).to(dtype)
    c.k, c.v = (torch.randn((T, Hkv, D), generator=gen).to(dtype) for _ in range(2))
    c.gen = gen
    return c


def attn_bounds(c, q, K, V, rows, sm_scale, mag, ref, exact_weights=False):
    """How far outputs (like ref) and log-sum-exps may be off.  Scores: fp32 sums of D products, each off by at most D + 8 half steps of
    the largest sum of magnitudes (products of bf16 are exact; their scale and distance to the reference are one rounding each).  Weights:
    twice that (numerator and sum), 8 half steps for the exponential and rescaling; sums of `rows` weights in fp32; weights rounded to the
    type; the result rounded to the type."""
    fin = lambda x: torch.nan_to_num(x.double(), nan=0.0, posinf=0.0, neginf=0.0).abs()
    # (an upper bound of sum |q k|: the largest rows' norms)
    score = abs(sm_scale) * float(fin(q).square().sum(-1).sqrt().max() * fin(K).square().sum(-1).sqrt().max())
    d_score = (c.D + 8) * U * score
    rel = 2 * (math.expm1(d_score) + 8 * U) + 2 * (rows + 16) * U
    step = half_step(c.dtype)
    out = mag * rel + 1e-30
    if not exact_weights:
        out = out + (0 if c.dtype == torch.float32 else mag * step * 1.01)
        out = out + ref.abs() * step * 1.01
    return out, d_score + (rows + 16) * U + 8 * U


def close(got, want, tol, what=""):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape
    fin = torch.isfinite(want)
    same = (got == want) | (got.isnan() & want.isnan())
    assert bool(same[~fin].all()), f"{what}: infinite and NaN elements differ"
    off = (got - want).abs()
    tol = torch.as_tensor(tol, dtype=torch.float64).expand_as(want)
    bad = fin & ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, by up to {float((off / tol)[bad].nan_to_num(nan=math.inf).max()):.3g} times what they may"
