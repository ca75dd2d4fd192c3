"""A cache held in pages, in a model's use of it: rows go in with their rotation, chunks of new tokens attend over it, selected rows too.

K and V are held as pages of some rows of every KV head, [pages, KV heads, rows of a page, D], and row n of sequence b is row n % page of
page table[b, n // page].  Sequence b has lens[b] rows, the last cu[b + 1] - cu[b] of them new in this call.

* append  new tokens' queries and keys are rotated by their positions, keys and values go to their rows.
* attn    causal attention of each sequence's new tokens over all of its rows: one token of a decode step, a chunk of a prompt, or both.
* sparse  decode attention over each head's list of selected rows, then the rows appended since the list was made.
"""
import math

import torch

own = False

DEV = "cuda"


# ---- the cases ------------------------------------------------------------------------------------
def listed():
    return [
        # Decoding a batch of 16: one token of every sequence, each at a length of its own.  Bound by the launch.
        dict(name="append_one_token", kind="append", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, rot=128, pairs=False, new="1*16", kept="16383*9,5000*7"),
        # A chunk of a long prompt, behind what the cache holds already: positions past 100K.
        dict(name="append_chunk_8k", kind="append", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, rot=128, pairs=False, new="8192", kept="122880"),
        # Ragged prompts in fp32, small heads of which half is rotated, by adjacent pairs.
        dict(name="append_ragged_f32", kind="append", dtype="f32", Hq=16, Hkv=4, D=64, page=16, rot=32, pairs=True, new="1,777,2501,0,64", kept="0,3,1025,40,9999"),
        # One token of the smallest configuration: latency.
        dict(name="attn_token_tiny_f32", kind="attn", dtype="f32", Hq=8, Hkv=8, D=64, page=16, window=0, new="1", kept="1023"),
        # A dense decode step of one sequence at 32K context, the headline shape.
        dict(name="attn_token_32k", kind="attn", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, window=0, new="1", kept="32767"),
        # A dense decode step of a batch.
        dict(name="attn_token_b16", kind="attn", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, window=0, new="1*16", kept="16383*8,16000*4,9001*4"),
        # A prompt of 8K tokens from the first one on.
        dict(name="attn_prompt_8k", kind="attn", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, window=0, new="8192", kept="0"),
        # A chunk of a long prompt over 64000 rows that are there already, 64 query heads on 8.
        dict(name="attn_chunk_over_64000", kind="attn", dtype="bf16", Hq=64, Hkv=8, D=128, page=128, window=0, new="1024", kept="64000"),
        # Prompts, a rest of one and decode tokens in one call, fp32, small heads, attention to the last 1500 rows.
        dict(name="attn_ragged_window_f32", kind="attn", dtype="f32", Hq=16, Hkv=4, D=64, page=16, window=1500, new="1,611,1,37,2049", kept="4100,5,77,3001,0"),
        # Selected rows of one sequence at 32K context: the headline shape.
        dict(name="sparse_32k", kind="sparse", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, B=1, N=32768, k=3277, tail=0),
        # A batch of 16, selected rows and those appended since.
        dict(name="sparse_b16", kind="sparse", dtype="bf16", Hq=32, Hkv=8, D=128, page=64, B=16, N=16384, k=2048, tail=7),
        # fp32, an odd length in small pages.
        dict(name="sparse_ragged_f32", kind="sparse", dtype="f32", Hq=16, Hkv=4, D=64, page=16, B=3, N=5003, k=701, tail=3),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        for x in w:
            most[c["kind"], x] = max(most.get((c["kind"], x), 0.0), w[x])
    while True:
        kind = rng.choice(("append", "attn", "attn", "attn", "sparse", "sparse"))
        d, hkv, g = rng.choice((64, 128, 128)), rng.choice((1, 2, 4, 8, 8, 8)), rng.choice((1, 2, 4, 4, 8))
        c = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")), Hq=g * hkv, Hkv=hkv, D=d, page=rng.choice((16, 16, 32, 64, 128, 256)))
        B = _log_int(rng, 1, 16)
        if kind == "sparse":
            n = _log_int(rng, 64, 1 << 17)
            k = max(1, min(8192, int(n * math.exp(rng.uniform(math.log(0.01), math.log(0.3))))))
            c.update(B=B, N=n, k=k, tail=rng.choice((0, 0, 1, 7, 15)))
            if B * hkv * n * d > 1 << 29:
                continue
        else:
            one = rng.random() < 0.4  # a decode step
            new = [1 if one or rng.random() < 0.1 else _log_int(rng, 1, 8192) for _ in range(B)]
            kept = [_log_int(rng, 1, 1 << 17) - 1 for _ in range(B)]
            c.update(new=",".join(map(str, new)), kept=",".join(map(str, kept)))
            if kind == "append":
                c.update(rot=rng.choice((d, d, d // 2)), pairs=rng.random() < 0.3)
            else:
                c["window"] = rng.choice((0, 0, 0, _log_int(rng, 16, 8192)))
            longest = max(n + k for n, k in zip(new, kept))
            if B * longest * hkv * d > 1 << 29 or (kind == "attn" and B * max(new) * c["Hq"] * longest > 1 << 32):
                continue
        w = work(c)
        if all(w[x] <= most[kind, x] for x in w):
            return c


def _counts(text):
    """"1*3,7" is [1, 1, 1, 7]."""
    got = []
    for part in text.split(","):
        n, _, times = part.partition("*")
        got += [int(n)] * int(times or 1)
    return got


def _elt(c):
    return 4 if c["dtype"] == "f32" else 2


def _torch_dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def work(c):
    g, e = c["Hq"] // c["Hkv"], _elt(c)
    if c["kind"] == "sparse":
        # g lists that do not depend on each other, each with a share p of the rows
        p = min(c["k"], c["N"] - c["tail"]) / c["N"]
        rows, distinct = p * c["N"] + c["tail"], c["N"] * (1 - (1 - p) ** g) + c["tail"]
        return {"bytes": c["B"] * (c["Hkv"] * distinct * 2 * c["D"] * e + c["Hq"] * (4 * p * c["N"] + c["D"] * (e + 4) + 4)),
                "flops": 4 * c["B"] * c["Hq"] * rows * c["D"]}
    new, kept = _counts(c["new"]), _counts(c["kept"])
    tokens = sum(new)
    if c["kind"] == "append":
        # queries and keys are read and written, keys twice (their rows, and in the tokens' order), values read and written
        return {"bytes": tokens * (2 * c["Hq"] + 5 * c["Hkv"]) * c["D"] * e, "flops": 3 * tokens * (c["Hq"] + c["Hkv"]) * c["rot"]}
    pairs = read = 0
    for n, k in zip(new, kept):
        w = c["window"] or n + k
        full = max(0, min(n, n + k - w))  # tokens that see a whole window; those before see 1, 2, ... more than is kept
        pairs += full * w + (n - full) * k + (n - full) * (n - full + 1) // 2
        read += (n + k - max(0, k + 1 - w)) if n else 0
    return {"bytes": read * c["Hkv"] * 2 * c["D"] * e + tokens * c["Hq"] * (2 * c["D"] * e + 4), "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---- inputs ---------------------------------------------------------------------------------------
def _lists(c, gen):
    """Ascending lists of k rows that favour some rows, as selections do, behind nothing that is in the dense range."""
    n = c["N"] - c["tail"]
    k = min(c["k"], n)
    score = torch.rand((c["B"], c["Hq"], n), generator=gen, device=DEV)
    return score.topk(k, dim=-1).indices.sort(-1).values.to(torch.int32).contiguous()


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    td, Hq, Hkv, D, page = _torch_dtype(c), c["Hq"], c["Hkv"], c["D"], c["page"]
    s = {"c": c}
    if c["kind"] == "sparse":
        new, lens = [0] * c["B"], [c["N"]] * c["B"]
    else:
        new, kept = _counts(c["new"]), _counts(c["kept"])
        lens = [n + k for n, k in zip(new, kept)]
    B, T = len(lens), sum(new)
    entries = max(1, max(-(-n // page) for n in lens))
    # pages are handed out in no order, as a server's that has run for a while; a sequence that is short names few of them
    pages = B * entries + 3
    s["table"] = torch.randperm(pages, generator=gen, device=DEV)[:B * entries].view(B, entries).to(torch.int32)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["cu"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=DEV)
    s["longest"], s["most_new"] = max(lens), max(new)
    s["K"], s["V"] = (torch.randn((pages, Hkv, page, D), generator=gen, device=DEV, dtype=td) for _ in range(2))
    if c["kind"] == "sparse":
        s["q"] = torch.randn((B, Hq, D), generator=gen, device=DEV).to(td)
        s["idx"] = _lists(c, gen)
        s["count"] = torch.full((B, Hq), s["idx"].shape[2], dtype=torch.int32, device=DEV)
        s["tail"] = (c["N"] - c["tail"], c["N"])
        s["out"], s["lse"] = torch.zeros((B, Hq, D), device=DEV), torch.zeros((B, Hq), device=DEV)
    elif c["kind"] == "append":
        # what a projection leaves: queries, keys and values of a token in one row
        qkv = torch.randn((T, (Hq + 2 * Hkv) * D), generator=gen, device=DEV).to(td).view(T, Hq + 2 * Hkv, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().to(DEV)
        s["q_out"] = torch.zeros((T, Hq, D), dtype=td, device=DEV)
        s["k_out"] = torch.zeros((T, Hkv, D), dtype=td, device=DEV)
    else:
        # queries that prefer some rows: logits of a standard deviation of 1.5
        s["q"] = (1.5 * torch.randn((T, Hq, D), generator=gen, device=DEV)).to(td)
        s["out"], s["lse"] = torch.zeros((T, Hq, D), dtype=td, device=DEV), torch.zeros((T, Hq), device=DEV)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps between calls: the cache's descriptors and the workspace."""
    from paper_2503_07518_amd import binding as tb

    c = s["c"]
    s["tb"] = tb
    s["cache"] = tb.PagedCache(s["K"], s["V"], s["table"])
    s["desc"] = tb.make_paged_desc(s["longest"], c["Hq"], s["cache"])
    if c["kind"] == "attn":
        s["ws"] = tb.new_workspace(tb.TB_OP_PAGED_ATTN, s["desc"], s["q"].shape[0])
    elif c["kind"] == "sparse":
        s["ws"] = tb.new_workspace(tb.TB_OP_ATTN, s["desc"], s["idx"].shape[2] + c["tail"])


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    c = s["c"]
    if own:
        tb = s["tb"]
        if c["kind"] == "append":
            tb.tb_append_paged_kv(s["desc"], s["cache"], s["q"], s["k"], s["v"], s["cu"], s["lens"], s["inv_freq"], s["q_out"], s["k_out"],
                                  interleaved=c["pairs"])
            return s["q_out"], s["k_out"], s["K"], s["V"]
        if c["kind"] == "attn":
            tb.tb_paged_attn(s["desc"], s["cache"], s["q"], s["cu"], s["lens"], s["most_new"], 1 / math.sqrt(c["D"]), s["out"], s["lse"], s["ws"],
                             window=c["window"])
            return s["out"], s["lse"]
        tb.tb_sparse_decode_attn_paged(s["desc"], s["cache"], s["q"], s["idx"], s["count"], s["idx"].shape[2], 1 / math.sqrt(c["D"]), s["out"],
                                       s["lse"], s["ws"], *s["tail"])
        return s["out"], s["lse"]
    return {"append": _plain_append, "attn": _plain_attn, "sparse": _plain_sparse}[c["kind"]](s)


def _tokens(s):
    """Of every new token: its sequence, its number among the sequence's new ones, its row in the cache."""
    t = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(s["cu"][1:].contiguous(), t, right=True)
    i = t - s["cu"][b]
    return b, i, s["lens"][b] - (s["cu"][b + 1] - s["cu"][b]) + i


def _rotate(x, cos, sin, pairs):
    """x [T, heads, rot] in 64 bits."""
    a, b = (x[..., 0::2], x[..., 1::2]) if pairs else x.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)


def _plain_append(s):
    c, page = s["c"], s["c"]["page"]
    b, _, p = _tokens(s)
    # (angles of far positions: 64 bits)
    angle = p.double()[:, None, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle), torch.sin(angle)
    q, k = (torch.cat((_rotate(x[..., :c["rot"]].double(), cos, sin, c["pairs"]), x[..., c["rot"]:].double()), -1).to(x.dtype) for x in (s["q"], s["k"]))
    at = s["table"][b, p // page].long()
    s["K"][at, :, p % page] = k
    s["V"][at, :, p % page] = s["v"]
    return q, k, s["K"], s["V"]


def _sequences(s, n):
    """The first n rows of every sequence, [B, KV heads, n, D] in 32 bits."""
    page = s["c"]["page"]
    p = torch.arange(n, device=DEV)
    at = s["table"][:, p // page].long()
    return (x[at, :, (p % page).expand_as(at)].transpose(1, 2).float().contiguous() for x in (s["K"], s["V"]))


def _softmax_rows(x, V):
    """Weights from logits (-inf: not attended), their sums, and the weighted rows of V."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, V) / total, (top + torch.log(total)).squeeze(-1)


def _plain_attn(s):
    c = s["c"]
    Hkv, D, g = c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    b, i, p = _tokens(s)
    B, most = s["lens"].shape[0], s["most_new"]
    q = torch.zeros((B, most, Hkv, g, D), device=DEV)
    q[b, i] = s["q"].float().view(-1, Hkv, g, D)
    row = torch.zeros((B, most), dtype=torch.int64, device=DEV)
    row[b, i] = p
    K, V = _sequences(s, s["longest"])
    q = q.permute(0, 2, 3, 1, 4).reshape(B, Hkv, g * most, D)
    x = torch.matmul(q, K.transpose(2, 3)).mul_(1 / math.sqrt(D)).view(B, Hkv, g, most, -1)
    n = torch.arange(s["longest"], device=DEV)
    hidden = n > row[..., None]
    if c["window"]:
        hidden = hidden | (n <= row[..., None] - c["window"])
    x.masked_fill_(hidden[:, None, None], -math.inf)
    out, lse = _softmax_rows(x.view(B, Hkv, g * most, -1), V)
    out = out.view(B, Hkv, g, most, D).permute(0, 3, 1, 2, 4)[b, i]
    lse = lse.view(B, Hkv, g, most).permute(0, 3, 1, 2)[b, i]
    return out.reshape(-1, c["Hq"], D).to(s["q"].dtype), lse.reshape(-1, c["Hq"])


def _plain_sparse(s):
    c, page = s["c"], s["c"]["page"]
    B, Hq, D = s["q"].shape
    tail = torch.arange(*s["tail"], device=DEV)
    rows = torch.cat((s["idx"].long(), tail.expand(B, Hq, -1)), -1)
    at = s["table"][torch.arange(B, device=DEV)[:, None, None], rows // page].long()
    kv = (torch.arange(Hq, device=DEV) // (Hq // c["Hkv"]))[:, None]
    K, V = (x[at, kv, rows % page].float() for x in (s["K"], s["V"]))
    x = torch.matmul(K, s["q"].float()[..., None]).squeeze(-1) * (1 / math.sqrt(D))
    out, lse = _softmax_rows(x[:, :, None], V)
    return out.squeeze(2), lse.squeeze(2)


# ---- the definition in 64 bits ----------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c, D, page = s["c"], case["D"], case["page"]
    g = c["Hq"] // c["Hkv"]
    lens, cu = s["lens"].tolist(), s["cu"].tolist()

    def rows_of(x, b, h, rows):
        return x[s["table"][b, rows // page].long(), h, rows % page].double()

    if c["kind"] == "append":
        K, V, half = s["K"].double(), s["V"].double(), c["rot"] // 2
        q, k = s["q"].double(), s["k"].double()
        for b, n in enumerate(lens):
            t = torch.arange(cu[b], cu[b + 1], device=DEV)
            p = torch.arange(n - t.numel(), n, device=DEV)
            # a pair of elements is a complex number, and the rotation a product with one of length 1
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), p[:, None].double() * s["inv_freq"].double())[:, None]
            for x in (q, k):
                r = x[t, :, :c["rot"]]
                if c["pairs"]:
                    z = torch.view_as_real(torch.view_as_complex(r.unflatten(-1, (half, 2)).contiguous()) * turn).flatten(-2)
                else:
                    z = torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous()) * turn
                    z = torch.cat((z.real, z.imag), -1)
                x[t, :, :c["rot"]] = z
            at = s["table"][b, p // page].long()
            K[at, :, p % page] = k[t]
            V[at, :, p % page] = s["v"][t].double()
        return q, k, K, V
    if c["kind"] == "sparse":
        out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
        tail = torch.arange(*s["tail"], device=DEV)
        for b in range(c["B"]):
            for h in range(c["Hq"]):
                rows = torch.cat((s["idx"][b, h, :int(s["count"][b, h])].long(), tail))
                x = rows_of(s["K"], b, h // g, rows) @ s["q"][b, h].double() / math.sqrt(D)
                lse[b, h] = torch.logsumexp(x, 0)
                out[b, h] = torch.exp(x - lse[b, h]) @ rows_of(s["V"], b, h // g, rows)
        return out, lse
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        t = torch.arange(cu[b], cu[b + 1], device=DEV)
        if not t.numel():
            continue
        rows, p = torch.arange(n, device=DEV), torch.arange(n - t.numel(), n, device=DEV)[:, None]
        seen = (rows <= p) & ((rows > p - c["window"]) if c["window"] else True)
        for hkv in range(c["Hkv"]):
            K, V = rows_of(s["K"], b, hkv, rows), rows_of(s["V"], b, hkv, rows)
            for h in range(hkv * g, hkv * g + g):
                x = (s["q"][t, h].double() @ K.T / math.sqrt(D)).masked_fill(~seen, -math.inf)
                lse[t, h] = torch.logsumexp(x, 1)
                out[t, h] = torch.exp(x - lse[t, h][:, None]) @ V
    return out, lse
