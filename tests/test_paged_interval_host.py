"""The interval loop over a cache in pages, where a call is refused or fails: its count of rows is that of the rows that are there.  Host only."""
import pytest
import torch

from paper_2503_07518_amd import binding as tb
from paper_2503_07518_amd.interval import PagedIntervalDecoder

F32, BF16 = torch.float32, torch.bfloat16
B, Hkv, Hq, D, d, PAGE, P = 2, 2, 8, 64, 16, 16, 3
CALLS = ("tb_append_paged_kv", "tb_paged_attn", "tb_project_keys", "tb_score", "tb_select_topk", "tb_expand_neighbors", "tb_sparse_decode_attn_paged")


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, which note their name and do nothing; a name in `fails` raises."""
    seen = type("Calls", (list,), {})()
    seen.fails = set()

    def stand_in(name):
        def call(*a, **k):
            if name in seen.fails:
                raise tb.TbError(tb.TB_ERR_UNSUPPORTED, name)
            seen.append(name)
        return call
    for name in CALLS:
        monkeypatch.setattr(tb, name, stand_in(name))
    monkeypatch.setattr(tb, "new_workspace", lambda *a, **k: torch.zeros(256, dtype=torch.uint8))
    return seen


def loop(**kw):
    pages = torch.zeros((9, Hkv, PAGE, D), dtype=BF16)
    cache = tb.PagedCache(pages, pages.clone(), torch.zeros((B, 4), dtype=torch.int32))
    kw = dict(dict(W=torch.zeros((1, D, d), dtype=BF16), Hq=Hq, k=4, P=P, radius=1), **kw)
    return PagedIntervalDecoder(cache, **kw)


def tokens(n, dtype=BF16):
    return [torch.zeros((B, n, h, D), dtype=dtype) for h in (Hq, Hkv, Hkv)]


def token(dtype=BF16):
    return [torch.zeros((B, h, D), dtype=dtype) for h in (Hq, Hkv, Hkv)] + [torch.zeros((B, Hq, d), dtype=dtype)]


def state(x):
    return x.N, x.n_waiting, x.N_pred, x.lens.tolist()


@pytest.mark.parametrize("fails", ["tb_append_paged_kv", "tb_paged_attn", "tb_project_keys"])
def test_a_prompt_that_fails(calls, fails):
    x = loop()
    x.prompt(*tokens(5))
    x.step(0, *token())
    x.step(1, *token())
    was = state(x)
    assert was == (7, 1, 6, [7, 7])
    calls.fails.add(fails)
    with pytest.raises(tb.TbError):
        x.prompt(*tokens(5))
    assert state(x) == was
    calls.fails.clear()
    x.prompt(*tokens(5))
    assert state(x) == (12, 0, 6, [12, 12])


@pytest.mark.parametrize("t", [3, 4])
@pytest.mark.parametrize("fails", CALLS)
def test_a_step_that_fails(calls, fails, t):
    """At every call of a step, one that predicts and one that does not; the step once more then leaves what it would have left."""
    x, y = loop(), loop()
    for z in (x, y):
        z.prompt(*tokens(5))
        for s in range(t):
            z.step(s, *token())
    was = state(x)
    calls.clear()
    y.step(t, *token())
    runs = list(calls)
    if fails not in runs:
        return
    calls.fails.add(fails)
    with pytest.raises(tb.TbError):
        x.step(t, *token())
    assert state(x) == was
    calls.fails.clear()
    x.step(t, *token())
    assert state(x) == state(y) == (was[0] + 1, t % P, was[0] + 1 if t % P == 0 else was[2], [was[0] + 1] * B)


def test_prompts_and_steps_of_another_type_or_shape(monkeypatch):
    def launched(*a, **k):
        raise RuntimeError("launched")
    monkeypatch.setattr(tb, "load_library", launched)
    monkeypatch.setattr(tb, "_lib", None)
    monkeypatch.setattr(tb, "new_workspace", lambda *a, **k: torch.zeros(256, dtype=torch.uint8))
    x = loop()
    q, k, v = tokens(3)
    for bad in (tokens(3, F32), (q, k.float(), v), (q, k, v.float()), (q[:1], k, v), (q, k[:, :2], v[:, :2]), (q[:, :, :4], k, v), (q, k[..., :32], v[..., :32])):
        with pytest.raises(AssertionError):
            x.prompt(*bad)
        assert state(x) == (0, 0, None, [0, 0])
    with pytest.raises(ValueError):
        x.prompt(*tokens(65))
    assert state(x) == (0, 0, None, [0, 0])


def test_a_step_before_any_prediction(calls):
    x = loop()
    x.prompt(*tokens(5))
    with pytest.raises(ValueError, match="prediction"):
        x.step(1, *token())
    assert state(x) == (5, 0, None, [5, 5])


@pytest.mark.parametrize("W", [torch.zeros((1, D, d)), torch.zeros((1, 2 * D, d), dtype=BF16), torch.zeros((1, D, 48), dtype=BF16), torch.zeros((1, D, 128), dtype=BF16),
                               torch.zeros((3, D, d), dtype=BF16), torch.zeros((D, d), dtype=BF16), torch.zeros((1, d, D), dtype=BF16).transpose(1, 2)])
def test_projections_of_another_type_or_shape(calls, W):
    with pytest.raises(AssertionError):
        loop(W=W)


@pytest.mark.parametrize("Hw", [1, Hkv])
def test_importance_queries_of_another_type_or_shape(calls, Hw):
    """The scores' kernel would read past their end, or as other numbers."""
    x = loop(W=torch.zeros((Hw, D, 32), dtype=BF16))
    x.prompt(*tokens(5))
    was = state(x)
    *qkv, _ = token()
    q_imp = torch.zeros((B, Hq, 32), dtype=BF16)
    for t in (0, 3):
        calls.clear()
        for bad in (q_imp.float(), q_imp[..., :16], q_imp[:1], q_imp[:, :4], torch.zeros((B, Hq, 64), dtype=BF16), torch.zeros((B, 1, 32), dtype=BF16),
                    torch.zeros((B, 32, Hq), dtype=BF16).transpose(1, 2)):
            with pytest.raises(AssertionError):
                x.step(t, *qkv, bad)
        assert not calls and state(x) == was
        x.step(t, *qkv, q_imp)
        assert calls
        x.step(t + 1, *qkv, None)
        was = state(x)
