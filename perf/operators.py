"""A cache held in microscaled 4-bit floating point: what fills it, scores it and attends over it, as timed cases.

The format is OCP's MXFP4: blocks of 32 elements along a row, each element a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1), each
block with a power of two (E8M0, 2^(byte - 127)).  Two elements share a byte, the even one in its low half.

* quantize   rows of K, V and the projected keys go into the cache, and are read back as the values it stands for: a new token of every
             sequence of a batch, a prompt, a chunk of one.
* score      importance of every cached token: importance queries times the projected keys.
* attn       decode attention over each head's list of rows, then the rows appended since the list was made.
* shared     the same with one list per sequence for all of its heads.
* dense      the same over all rows of the cache.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32


# ---- the cases ------------------------------------------------------------------------------------
def listed():
    return [
        # Decoding a batch of 16: the new token's K, V and projected key of every KV head.  Bound by launches.
        dict(name="quantize_one_token", kind="quantize", dtype="bf16", B=16, Hkv=8, D=128, Dimp=32, rows=1),
        # After a prompt of 32K tokens: the whole layer's cache.
        dict(name="quantize_prompt_32k", kind="quantize", dtype="bf16", B=1, Hkv=8, D=128, Dimp=32, rows=32768),
        # A chunk of prompts in fp32, odd in length, small heads.
        dict(name="quantize_chunk_f32", kind="quantize", dtype="f32", B=3, Hkv=4, D=64, Dimp=64, rows=5003),
        # Scores of the smallest configuration's size: latency.
        dict(name="score_tiny_f32", kind="score", dtype="f32", B=1, Hq=8, Hkv=8, N=1024, Dimp=32),
        # One sequence at 32K context, the headline shape.
        dict(name="score_32k", kind="score", dtype="bf16", B=1, Hq=32, Hkv=8, N=32768, Dimp=32),
        # Long contexts on a model with 64 query heads.
        dict(name="score_128k_64heads", kind="score", dtype="bf16", B=4, Hq=64, Hkv=8, N=131072, Dimp=32),
        # The smallest configuration's attention.
        dict(name="attn_tiny_f32", kind="attn", dtype="f32", B=1, Hq=8, Hkv=8, D=64, N=1024, k=128, tail=0, widened=False),
        # Interactive decoding at 32K context, a tenth of the rows.
        dict(name="attn_32k", kind="attn", dtype="bf16", B=1, Hq=32, Hkv=8, D=128, N=32768, k=3277, tail=0, widened=False),
        # A serving batch of 16 sequences at 16K context.
        dict(name="attn_batch16_16k", kind="attn", dtype="bf16", B=16, Hq=32, Hkv=8, D=128, N=16384, k=2048, tail=0, widened=False),
        # A step inside a prediction interval: lists widened by their neighbours, so of uneven length, and the 7 rows since.
        dict(name="attn_reuse_64k", kind="attn", dtype="bf16", B=4, Hq=32, Hkv=8, D=128, N=65536, k=4096, tail=7, widened=True),
        # The variant with one importance head: one list per sequence for all heads.
        dict(name="shared_32k", kind="shared", dtype="bf16", B=4, Hq=32, Hkv=8, D=128, N=32768, k=3661, tail=0),
        # Dense attention over every cached row, 64 query heads on 8, a small batch at an odd length.
        dict(name="dense_ragged_64heads", kind="dense", dtype="bf16", B=3, Hq=64, Hkv=8, D=128, N=20011),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), work(c)["bytes"])
    most["shared"] = most["dense"] = max(most["shared"], most["dense"])
    while True:
        kind = rng.choice(("quantize", "score", "attn", "attn", "shared", "dense"))
        dtype, hkv, g = rng.choice(("bf16", "bf16", "bf16", "f32")), rng.choice((1, 2, 4, 8, 8, 8)), rng.choice((1, 2, 4, 4, 8))
        d, dimp = rng.choice((64, 128, 128)), rng.choice((32, 32, 64))
        if kind == "quantize":
            c = dict(kind=kind, dtype=dtype, B=_log_int(rng, 1, 16), Hkv=hkv, D=d, Dimp=dimp, rows=_log_int(rng, 1, 32768))
        elif kind == "score":
            c = dict(kind=kind, dtype=dtype, B=_log_int(rng, 1, 16), Hq=g * hkv, Hkv=hkv, N=_log_int(rng, 1, 1 << 18), Dimp=dimp)
        else:
            n = _log_int(rng, 64, 1 << 17)
            k = max(1, min(8192, int(n * math.exp(rng.uniform(math.log(0.01), math.log(0.3))))))
            c = dict(kind=kind, dtype=dtype, B=_log_int(rng, 1, 16), Hq=g * hkv, Hkv=hkv, D=d, N=n)
            if kind != "dense":
                c.update(k=k, tail=rng.choice((0, 0, 1, 7, 15)))
            if kind == "attn":
                c["widened"] = rng.random() < 0.3
            if c["B"] * c["Hkv"] * n * d > 1 << 29:
                continue
        if work(c)["bytes"] <= most[kind]:
            return c


def _elt(c):
    return 4 if c["dtype"] == "f32" else 2


def _torch_dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _row_bytes(inner):
    return inner // 2 + inner // BLOCK


def work(c):
    if c["kind"] == "quantize":
        n = c["B"] * c["Hkv"] * c["rows"]
        per_row = 2 * c["D"] + c["Dimp"]
        return {"bytes": n * (2 * per_row * _elt(c) + _row_bytes(per_row)), "flops": 4 * n * per_row}
    if c["kind"] == "score":
        return {"bytes": c["B"] * (c["Hkv"] * c["N"] * _row_bytes(c["Dimp"]) + c["Hq"] * (4 * c["N"] + c["Dimp"] * _elt(c))),
                "flops": 2 * c["B"] * c["Hq"] * c["N"] * c["Dimp"]}
    g, n = c["Hq"] // c["Hkv"], c["N"]
    if c["kind"] == "dense":
        rows = distinct = n
        entries = 0
    else:
        # a list and its neighbours keep 1 - (1 - p)^3 of the rows; g lists that do not depend on each other, the share that one of them has
        p = min(c["k"], n) / n
        p = 1 - (1 - p) ** 3 if c.get("widened") else p
        rows = p * n + c["tail"]
        distinct = (n * (1 - (1 - p) ** g) if c["kind"] == "attn" else p * n) + c["tail"]
        entries = c["B"] * (c["Hq"] if c["kind"] == "attn" else 1) * p * n
    return {"bytes": c["B"] * c["Hkv"] * distinct * 2 * _row_bytes(c["D"]) + 4 * entries + c["B"] * c["Hq"] * (c["D"] * (_elt(c) + 4) + 4),
            "flops": 4 * c["B"] * c["Hq"] * rows * c["D"]}


# ---- the format in elementary operations ------------------------------------------------------------
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_tables = {}


def _decode_tables(dev):
    """Both values of every byte of codes [256, 2], and the factor of every scale byte [256]."""
    if dev not in _tables:
        e2m1 = torch.tensor(_MAGNITUDES + tuple(-m for m in _MAGNITUDES), dtype=torch.float32)
        byte = torch.arange(256)
        scale = torch.ldexp(torch.ones(256, dtype=torch.float64), torch.arange(256) - 127).float()
        scale[255] = math.nan
        _tables[dev] = (torch.stack((e2m1[byte & 15], e2m1[byte >> 4]), -1).to(dev), scale.to(dev))
    return _tables[dev]


def _decode(codes, scales):
    """codes [..., inner / 2], scales [..., inner / 32] -> fp32 [..., inner]"""
    pair, factor = _decode_tables(codes.device)
    lead = codes.shape[:-1]
    v = pair.index_select(0, codes.reshape(-1).int()).view(*lead, -1, BLOCK)
    v *= factor.index_select(0, scales.reshape(-1).int()).view(*lead, -1, 1)
    return v.view(*lead, -1)


def _encode(x):
    """[..., inner] -> codes [..., inner / 2], scales [..., inner / 32].  The block's power of two is that of its largest element, less
    the 2 of the largest code's; elements go to the nearest code, halves to the even one, and past 6 to 6."""
    lead, inner = x.shape[:-1], x.shape[-1]
    blocks = x.double().view(*lead, inner // BLOCK, BLOCK)
    amax = blocks.abs().amax(-1, keepdim=True)
    exponent = torch.frexp(amax)[1].sub_(3).clamp_(min=-127)
    exponent = torch.where(amax > 0, exponent, torch.full_like(exponent, -127))
    fine = torch.isfinite(amax)
    exponent = torch.where(fine, exponent, torch.full_like(exponent, 128))
    # (the unit as a number in 64 bits by its exponent field: the device's power function rounds some powers of two)
    y = blocks * (1023 - exponent.long() << 52).view(torch.float64)
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for half, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= half) if up else (a > half)
    code |= (y < 0).to(torch.uint8) << 3
    code = code.view(*lead, inner // 2, 2)
    return code[..., 0] | code[..., 1] << 4, (exponent + 127).to(torch.uint8).view(*lead, inner // BLOCK)


# ---- inputs ---------------------------------------------------------------------------------------
def _fill(codes, scales, gen):
    """A cache as quantised K or V rows leave it (a head at a time: the rows themselves are not kept)."""
    B, H, n, half = codes.shape
    for b in range(B):
        codes[b], scales[b] = _encode(torch.randn((H, n, 2 * half), generator=gen, device=DEV))


def _lists(c, heads, gen):
    """Ascending lists of k rows a head, drawn apart; widened: with both neighbours, so that their lengths differ."""
    n, k = c["N"] - c["tail"], min(c["k"], c["N"] - c["tail"])
    idx, most, count = [], 0, []
    for _ in range(c["B"]):
        at = torch.rand((heads, n), generator=gen, device=DEV).topk(k, dim=1).indices
        if c.get("widened"):
            keep = torch.zeros((heads, n + 2), dtype=torch.bool, device=DEV)
            for r in (0, 1, 2):
                keep.scatter_(1, at + r, True)
            keep = keep[:, 1:-1]
            count.append(keep.sum(1))
            idx.append(torch.argsort(keep.logical_not().to(torch.uint8), dim=1, stable=True)[:, :min(n, 3 * k)])
        else:
            count.append(torch.full((heads,), k, device=DEV))
            idx.append(at.sort(dim=1).values)
    return torch.stack(idx).int().contiguous(), torch.stack(count).int().contiguous()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    td, B, Hkv = _torch_dtype(c), c["B"], c["Hkv"]
    s = dict(c=c)

    def rows_of(n, inner):
        return (torch.zeros((B, Hkv, n, inner // 2), dtype=torch.uint8, device=DEV),
                torch.zeros((B, Hkv, n, inner // BLOCK), dtype=torch.uint8, device=DEV))

    def side_by_side(n, inner):
        """K and V of a token next to each other, as a cache of this format is laid out."""
        codes = torch.zeros((B, Hkv, n, 2, inner // 2), dtype=torch.uint8, device=DEV)
        scales = torch.zeros((B, Hkv, n, 2, inner // BLOCK), dtype=torch.uint8, device=DEV)
        return (codes[:, :, :, 0], scales[:, :, :, 0]), (codes[:, :, :, 1], scales[:, :, :, 1])

    if c["kind"] == "quantize":
        n = c["rows"]
        # rows of differing size, as heads and channels of a cache have
        s["K"], s["V"], s["Kimp"] = (
            (torch.randn((B, Hkv, n, i), generator=gen, device=DEV) * torch.randn((1, Hkv, 1, i), generator=gen, device=DEV).exp()).to(td)
            for i in (c["D"], c["D"], c["Dimp"]))
        s["Kq"], s["Vq"] = side_by_side(n, c["D"])
        s["Kimpq"] = rows_of(n, c["Dimp"])
        s["out"] = [torch.zeros_like(s[x]) for x in ("K", "V", "Kimp")]
    elif c["kind"] == "score":
        s["Kimpq"] = rows_of(c["N"], c["Dimp"])
        _fill(*s["Kimpq"], gen)
        s["q_imp"] = torch.randn((B, c["Hq"], c["Dimp"]), generator=gen, device=DEV).to(td)
        s["scores"] = torch.zeros((B, c["Hq"], (c["N"] + 3) // 4 * 4), device=DEV)
    else:
        s["Kq"], s["Vq"] = side_by_side(c["N"], c["D"])
        _fill(*s["Kq"], gen)
        _fill(*s["Vq"], gen)
        s["q"] = torch.randn((B, c["Hq"], c["D"]), generator=gen, device=DEV).to(td)
        if c["kind"] == "dense":
            s["idx"] = s["count"] = None
            s["most"], s["tail"] = 0, (0, c["N"])
        else:
            s["idx"], s["count"] = _lists(c, c["Hq"] if c["kind"] == "attn" else 1, gen)
            s["most"], s["tail"] = s["idx"].shape[2], (c["N"] - c["tail"], c["N"])
        s["o"], s["lse"] = torch.zeros((B, c["Hq"], c["D"]), device=DEV), torch.zeros((B, c["Hq"]), device=DEV)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps between calls: the cache's descriptors and the workspace."""
    from paper_2503_07518_amd import binding as tb

    c = s["c"]
    s["tb"] = tb
    for x in ("Kq", "Vq", "Kimpq"):
        if x in s:
            s[x + "_rows"] = tb.MxRows(*s[x])
    if c["kind"] == "quantize":
        # (no query heads take part in filling a cache)
        s["desc"] = tb.make_desc(c["rows"], c["Hkv"], K=s["K"], V=s["V"], Kimp=s["Kimp"])
        s["back"] = tb.make_desc(c["rows"], c["Hkv"], K=s["out"][0], V=s["out"][1], Kimp=s["out"][2])
    elif c["kind"] == "score":
        s["desc"] = tb.make_mx_desc(c["N"], c["Hq"], _torch_dtype(c), Kimp=s["Kimpq_rows"])
    else:
        s["desc"] = tb.make_mx_desc(c["N"], c["Hq"], _torch_dtype(c), K=s["Kq_rows"])
        s["ws"] = tb.new_workspace(tb.TB_OP_ATTN_MX, s["desc"], s["most"] + s["tail"][1] - s["tail"][0])


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    kind = s["c"]["kind"]
    if own:
        return _run_own(s, kind)
    if kind == "quantize":
        return [_decode(*_encode(s[x].float())).to(s[x].dtype) for x in ("K", "V", "Kimp")]
    if kind == "score":
        keys = _decode(*s["Kimpq"])
        B, Hkv = keys.shape[:2]
        q = s["q_imp"].float().view(B, Hkv, -1, keys.shape[3])
        return torch.matmul(q, keys.transpose(2, 3)).view(B, -1, keys.shape[2])
    return _plain_attention(s, kind)


def _run_own(s, kind):
    tb = s["tb"]
    if kind == "quantize":
        n = s["c"]["rows"]
        tb.tb_quantize_mx(s["desc"], s["K"], s["V"], s["Kimp"], 0, s["Kq_rows"], s["Vq_rows"], s["Kimpq_rows"], 0, n)
        tb.tb_dequantize_mx(s["back"], s["Kq_rows"], s["Vq_rows"], s["Kimpq_rows"], 0, *s["out"], 0, n)
        return s["out"]
    if kind == "score":
        tb.tb_score_mx(s["desc"], s["q_imp"], s["Kimpq_rows"], 1.0, s["scores"])
        return s["scores"][:, :, :s["c"]["N"]]
    attend = tb.tb_sparse_decode_attn_mx if kind == "attn" else tb.tb_sparse_decode_attn_shared_mx
    attend(s["desc"], s["q"], s["Kq_rows"], s["Vq_rows"], s["idx"], s["count"], s["most"], 1 / math.sqrt(s["c"]["D"]), s["o"], s["lse"], s["ws"],
           *s["tail"])
    return s["o"], s["lse"]


def _listed_rows(idx, count, tail):
    """Row numbers [B, heads, slots] of the lists and the range behind them, and which slots there are."""
    slot = torch.arange(idx.shape[2] + tail[1] - tail[0], device=idx.device)
    behind = slot - count[..., None]
    listed_ = behind < 0
    rows = torch.where(listed_, torch.nn.functional.pad(idx, (0, tail[1] - tail[0])), tail[0] + behind)
    there = rows < tail[1] if tail[1] > tail[0] else listed_
    return torch.where(there, rows, 0), there


def _plain_attention(s, kind):
    c, q = s["c"], s["q"].float()
    B, Hq, D = q.shape
    Hkv, g, n = c["Hkv"], c["Hq"] // c["Hkv"], c["N"]
    if kind == "dense":
        K, V = _decode(*s["Kq"]), _decode(*s["Vq"])
        there = None
    else:
        rows, there = _listed_rows(s["idx"], s["count"], s["tail"])
        heads = rows.shape[1]
        if kind == "shared":
            rows = rows.expand(B, Hkv, -1)
            kv = torch.arange(Hkv, device=q.device)
        else:
            kv = torch.arange(heads, device=q.device) // g
        b = torch.arange(B, device=q.device)[:, None, None]
        K, V = (_decode(x[0][b, kv[:, None], rows], x[1][b, kv[:, None], rows]) for x in (s["Kq"], s["Vq"]))
    q = q.view(B, K.shape[1], -1, D)  # [B, heads that have rows of their own, query heads that share them, D]
    x = torch.matmul(q, K.transpose(2, 3)) * (1 / math.sqrt(D))
    if there is not None:
        x = torch.where(there[:, :, None, :], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    return (torch.matmul(e, V) / total).view(B, Hq, D), (top + torch.log(total)).view(B, Hq)


# ---- the definition in 64 bits ----------------------------------------------------------------------
def _power(e):
    """2^e for whole e (the device's power function rounds some of them)."""
    table = torch.tensor([math.ldexp(1.0, i) for i in range(-160, 160)], dtype=torch.float64)
    return table.to(e.device)[e.long() + 160]


def _stands_for(codes, scales):
    """Element by element, from the bits."""
    nibble = torch.stack((codes % 16, codes // 16), -1).flatten(-2).double()
    sign, e, m = (nibble >= 8).double(), (nibble % 8) // 2, nibble % 2
    magnitude = torch.where(e > 0, (1 + m / 2) * _power(e - 1), m / 2)
    return (1 - 2 * sign) * magnitude * _power(scales.long() - 127).repeat_interleave(BLOCK, -1)


def _nearest(x):
    """The values that rows go to."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    largest = b.abs().amax(-1, keepdim=True)
    unit = _power((torch.floor(torch.log2(largest.clamp(min=2.0 ** -126))) - 2).clamp(min=-127))
    unit = torch.where(unit * 8 <= largest, unit * 2, unit)  # (a logarithm that was rounded down)
    unit = torch.where((unit * 4 > largest) & (unit > 2.0 ** -127), unit / 2, unit)  # (or up)
    y = b / unit
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return ((torch.round(y / step) * step).clamp(-6, 6) * unit).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "quantize":
        return [_nearest(s[x]) for x in ("K", "V", "Kimp")]
    g = c["Hq"] // c["Hkv"]
    if c["kind"] == "score":
        got = torch.empty((c["B"], c["Hq"], c["N"]), dtype=torch.float64, device=DEV)
        for b in range(c["B"]):
            keys = _stands_for(s["Kimpq"][0][b], s["Kimpq"][1][b])
            for h in range(c["Hq"]):
                got[b, h] = keys[h // g] @ s["q_imp"][b, h].double()
        return got
    out = torch.zeros((c["B"], c["Hq"], c["D"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros((c["B"], c["Hq"]), dtype=torch.float64, device=DEV)
    tail = torch.arange(*s["tail"], device=DEV)
    for b in range(c["B"]):
        for h in range(c["Hq"]):
            rows = tail
            if s["idx"] is not None:
                at = h if c["kind"] == "attn" else 0
                rows = torch.cat((s["idx"][b, at, :int(s["count"][b, at])].long(), tail))
            K, V = (_stands_for(x[0][b, h // g][rows], x[1][b, h // g][rows]) for x in (s["Kq"], s["Vq"]))
            logits = K @ s["q"][b, h].double() / math.sqrt(c["D"])
            lse[b, h] = torch.logsumexp(logits, 0)
            out[b, h] = torch.exp(logits - lse[b, h]) @ V
    return out, lse
