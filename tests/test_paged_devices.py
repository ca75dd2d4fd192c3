"""The kernels of a paged cache run on the current device: a call with any of its tensors on another GPU is refused, whichever it is.
Stand-ins for tensors, no GPU needed."""
import types

import pytest
import torch

from paper_2503_07518_amd import binding as tb

HERE, OTHER, HOST = 2, 1, -1


class Tensor:
    def __init__(self, device, shape, dtype=torch.float32):
        self.where, self.shape, self.dtype, self.nbytes = device, torch.Size(shape), dtype, 4096

    def get_device(self):
        return self.where

    def data_ptr(self):
        return 0x10000

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def stride(self, dim=None):
        st = [1]
        for n in self.shape[:0:-1]:
            st.insert(0, st[0] * n)
        return tuple(st) if dim is None else st[dim]

    device = property(lambda self: self.where)


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, which all do nothing here."""
    seen = []
    names = ("tb_append_paged_kv", "tb_paged_attn", "tb_sparse_decode_attn_paged")
    monkeypatch.setattr(tb, "_lib", types.SimpleNamespace(**{n: lambda *a, n=n: seen.append((n, a[-1])) or 0 for n in names}))
    monkeypatch.setattr(tb, "_get_device", lambda: HERE)
    monkeypatch.setattr(tb, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(tb, "_several_devices", True)
    return seen


INT = torch.int32
SHAPES = {
    "tb_append_paged_kv": dict(q=((4, 8, 64),), k=((4, 2, 64),), v=((4, 2, 64),), cu=((3,), INT), lens=((2,), INT), inv_freq=((32,),), q_out=((4, 8, 64),),
                               k_out=((4, 2, 64),), positions=((4,), INT)),
    "tb_paged_attn": dict(q=((4, 8, 64),), cu=((3,), INT), lens=((2,), INT), out=((4, 8, 64),), lse=((4, 8),), ws=((4096,), torch.uint8)),
    "tb_sparse_decode_attn_paged": dict(q=((2, 8, 64),), idx=((2, 8, 5), INT), count=((2, 8), INT), out=((2, 8, 64),), lse=((2, 8),), ws=((4096,), torch.uint8)),
}


def call(name, at):
    """`at`: a function from an argument's name to its device."""
    cache = tb.PagedCache(*(Tensor(at("cache"), (9, 2, 16, 64)) for _ in "KV"), Tensor(at("cache"), (2, 4), INT))
    d = tb.make_paged_desc(64, 8, cache)
    t = {n: Tensor(at(n), *x) for n, x in SHAPES[name].items()}
    if name == "tb_append_paged_kv":
        tb.tb_append_paged_kv(d, cache, **t)
    elif name == "tb_paged_attn":
        tb.tb_paged_attn(d, cache, max_new=4, sm_scale=1.0, **t)
    else:
        tb.tb_sparse_decode_attn_paged(d, cache, max_count=5, sm_scale=1.0, **t)


@pytest.mark.parametrize("name", SHAPES)
def test_tensors_on_another_device(calls, name):
    call(name, lambda n: HERE)
    assert calls == [(name, 1000 + HERE)]
    for wrong in ("cache", *SHAPES[name]):
        calls.clear()
        with pytest.raises(ValueError, match="current device"):
            call(name, lambda n: OTHER if n == wrong else HERE)
        assert not calls


def test_a_cache_on_two_devices():
    with pytest.raises(ValueError):
        tb.PagedCache(Tensor(HERE, (9, 2, 16, 64)), Tensor(OTHER, (9, 2, 16, 64)), Tensor(HERE, (2, 4), INT))
    with pytest.raises(ValueError):
        tb.PagedCache(Tensor(HERE, (9, 2, 16, 64)), Tensor(HERE, (9, 2, 16, 64)), Tensor(HOST, (2, 4), INT))
