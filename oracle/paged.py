"""The operators of a cache in pages, from their definitions, in 64 bits and one token at a time (test infrastructure).

Everything is a torch tensor on the CPU; K, V [pages, Hkv, page, D], table [B, entries], cu [B + 1], lens [B] as in include/tokenbutler.h."""
import math
from fractions import Fraction

import torch

PI = Fraction("3.141592653589793238462643383279502884197169399375105820974944592307812")


def place(table, b, n, page, pages):
    """Page and row in it of row n of sequence b; None in a hole."""
    p = int(table[b, n // page])
    return (p, n % page) if 0 <= p < pages else None


def tokens(cu, lens, N, max_new=None):
    """(t, b, row) of the tokens that take part."""
    for b in range(len(lens)):
        first, n = int(cu[b]), int(cu[b + 1] - cu[b])
        for i in range(n if max_new is None else min(n, max_new)):
            row = int(lens[b]) - n + i
            if 0 <= row < N:
                yield first + i, b, row


def cos_sin(position, inv_freq):
    """Of position * inv_freq: the product and what is left of its last turn are exact, whatever the position."""
    angle = Fraction(position) * Fraction(inv_freq)
    left = float(angle - round(angle / (2 * PI)) * 2 * PI)
    return math.cos(left), math.sin(left)


def append(q, k, v, K, V, table, cu, lens, N, inv_freq, interleaved, positions=None):
    """Returns rotated q and k, and K and V with their new rows, all in 64 bits; tokens that take no part keep what they had as NaN."""
    page, pages = K.shape[2], K.shape[0]
    q_out, k_out = torch.full(q.shape, math.nan, dtype=torch.float64), torch.full(k.shape, math.nan, dtype=torch.float64)
    K, V = K.double(), V.double()
    rot = 0 if inv_freq is None else 2 * len(inv_freq)
    for t, b, row in tokens(cu, lens, N):
        at = row if positions is None else int(positions[t])
        for x, out in ((q, q_out), (k, k_out)):
            y = x[t].double().clone()
            for i in range(rot // 2):
                lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
                c, s = cos_sin(at, float(inv_freq[i]))
                y[:, lo], y[:, hi] = x[t, :, lo].double() * c - x[t, :, hi].double() * s, x[t, :, hi].double() * c + x[t, :, lo].double() * s
            out[t] = y
        where = place(table, b, row, page, pages)
        if where:
            K[where[0], :, where[1]] = k_out[t]
            V[where[0], :, where[1]] = v[t].double()
    return q_out, k_out, K, V


def attend(q, K, V, rows, sm_scale):
    """One query [D] over rows K, V [n, D] in 64 bits: output, log-sum-exp, and the mean of |V| by the weights."""
    if len(rows) == 0:
        return torch.zeros(K.shape[-1], dtype=torch.float64), -math.inf, torch.zeros(K.shape[-1], dtype=torch.float64)
    x = (K @ q) * sm_scale
    if bool((x == -math.inf).all()):
        return torch.zeros(K.shape[-1], dtype=torch.float64), -math.inf, torch.zeros(K.shape[-1], dtype=torch.float64)
    lse = torch.logsumexp(x, 0)
    w = torch.exp(x - lse)
    return w @ V, float(lse), w @ V.abs()


def gather(X, table, b, hkv, rows):
    """Rows of a sequence [n, D] in 64 bits, those in holes left out, and their numbers."""
    page, pages = X.shape[2], X.shape[0]
    at = [(place(table, b, n, page, pages)) for n in rows]
    kept = [n for n, p in zip(rows, at) if p]
    at = [p for p in at if p]
    if not at:
        return torch.zeros((0, X.shape[3]), dtype=torch.float64), kept
    return X[torch.tensor([p for p, _ in at]), hkv, torch.tensor([r for _, r in at])].double(), kept


def attn(q, K, V, table, cu, lens, N, sm_scale, window=0, max_new=None):
    """Outputs, log-sum-exps and mean |V| of the new tokens [T, Hq, ...] (NaN: takes no part)."""
    T, Hq, D = q.shape
    g = Hq // K.shape[1]
    out, mag = (torch.full((T, Hq, D), math.nan, dtype=torch.float64) for _ in range(2))
    lse = torch.full((T, Hq), math.nan, dtype=torch.float64)
    for b in range(len(lens)):
        mine = [(t, row) for t, bb, row in tokens(cu, lens, N, max_new) if bb == b]
        if not mine:
            continue
        last = max(row for _, row in mine)
        for hkv in range(K.shape[1]):
            Kb, kept = gather(K, table, b, hkv, range(last + 1))
            Vb, _ = gather(V, table, b, hkv, range(last + 1))
            number = torch.tensor(kept, dtype=torch.int64)
            for t, row in mine:
                seen = (number <= row) & (number > row - window if window else torch.ones(len(kept), dtype=torch.bool))
                for h in range(hkv * g, hkv * g + g):
                    out[t, h], lse[t, h], mag[t, h] = attend(q[t, h].double(), Kb[seen], Vb[seen], number[seen], sm_scale)
    return out, lse, mag


def sparse(q, K, V, table, idx, count, tail, sm_scale):
    """Outputs, log-sum-exps and mean |V| [B, Hq, ...] over each head's list and the dense range."""
    B, Hq, D = q.shape
    g = Hq // K.shape[1]
    out, mag, lse = torch.zeros((B, Hq, D), dtype=torch.float64), torch.zeros((B, Hq, D), dtype=torch.float64), torch.zeros((B, Hq), dtype=torch.float64)
    for b in range(B):
        for h in range(Hq):
            rows = idx[b, h, :int(count[b, h])].tolist() + list(range(*tail))
            Kb, kept = gather(K, table, b, h // g, rows)
            Vb, _ = gather(V, table, b, h // g, rows)
            out[b, h], lse[b, h], mag[b, h] = attend(q[b, h].double(), Kb, Vb, kept, sm_scale)
    return out, lse, mag
