"""The kernels of the 4-bit cache run on the current device: a call with any of its tensors on another GPU is refused, whichever it is.
Stand-ins for tensors, no GPU needed."""
import types

import pytest
import torch

from paper_2503_07518_amd import binding as tb

HERE, OTHER, HOST = 2, 1, -1


class Tensor:
    dtype, nbytes = torch.float32, 4096

    def __init__(self, device):
        self.where = device

    def get_device(self):
        return self.where

    def data_ptr(self):
        return 0x10000

    def is_contiguous(self):
        return True

    def stride(self, dim):
        return 1 if dim == -1 else 64


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, which all do nothing here."""
    seen = []
    names = ("tb_quantize_mx", "tb_dequantize_mx", "tb_score_mx", "tb_sparse_decode_attn_mx", "tb_sparse_decode_attn_shared_mx")
    monkeypatch.setattr(tb, "_lib", types.SimpleNamespace(**{n: lambda *a, n=n: seen.append((n, a[-1])) or 0 for n in names}))
    monkeypatch.setattr(tb, "_get_device", lambda: HERE)
    monkeypatch.setattr(tb, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(tb, "_several_devices", True)
    return seen


def rows(device):
    r = tb.MxRows(torch.zeros((1, 1, 4, 32), dtype=torch.uint8), torch.zeros((1, 1, 4, 2), dtype=torch.uint8))
    r.device = device
    return r


def call(name, at):
    """`at`: a function from an argument's name to its device."""
    d = tb.tb_cache_desc()
    t, m = lambda n: Tensor(at(n)), lambda n: rows(at(n))
    if name == "tb_quantize_mx":
        tb.tb_quantize_mx(d, t("K"), t("V"), t("Kimp"), 0, m("Kq"), m("Vq"), m("Kimpq"), 0, 1)
    elif name == "tb_dequantize_mx":
        tb.tb_dequantize_mx(d, m("Kq"), m("Vq"), m("Kimpq"), 0, t("K"), t("V"), t("Kimp"), 0, 1)
    elif name == "tb_score_mx":
        tb.tb_score_mx(d, t("q_imp"), m("Kimp"), 1.0, t("scores"))
    else:
        getattr(tb, name)(d, t("q"), m("K"), m("V"), t("idx"), t("count"), 8, 1.0, t("out"), t("lse"), t("ws"))


ARGS = {"tb_quantize_mx": ("K", "V", "Kimp", "Kq", "Vq", "Kimpq"), "tb_dequantize_mx": ("K", "V", "Kimp", "Kq", "Vq", "Kimpq"),
        "tb_score_mx": ("q_imp", "Kimp", "scores"), "tb_sparse_decode_attn_mx": ("q", "K", "V", "idx", "count", "out", "lse", "ws"),
        "tb_sparse_decode_attn_shared_mx": ("q", "K", "V", "idx", "count", "out", "lse", "ws")}


@pytest.mark.parametrize("name,which", [(n, a) for n, args in ARGS.items() for a in args])
def test_any_tensor_on_another_device(calls, name, which):
    with pytest.raises(ValueError, match="cuda:1"):
        call(name, lambda n: OTHER if n == which else HERE)
    assert not calls
    call(name, lambda n: HOST if n == which else HERE)  # (host memory that the device reaches)
    call(name, lambda n: HERE)
    assert calls == [(name, 1000 + HERE)] * 2


@pytest.mark.parametrize("name", ["tb_sparse_decode_attn_mx", "tb_sparse_decode_attn_shared_mx"])
def test_calls_without_lists_and_lse(calls, name):
    d = tb.tb_cache_desc()
    getattr(tb, name)(d, Tensor(HERE), rows(HERE), rows(HERE), None, None, 0, 1.0, Tensor(HERE), None, Tensor(HERE), 0, 4)
    for n in ("tb_quantize_mx", "tb_dequantize_mx"):
        a = ([Tensor(HERE), None, None], [rows(HERE), None, None])
        x, y = a if n == "tb_quantize_mx" else a[::-1]
        getattr(tb, n)(d, *x, 0, *y, 0, 1)
    assert len(calls) == 3


def test_rows_name_the_device_of_both_arrays(monkeypatch):
    codes, scales = torch.zeros((1, 1, 4, 32), dtype=torch.uint8), torch.zeros((1, 1, 4, 2), dtype=torch.uint8)
    where = {}
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: where[t.data_ptr()])
    for c, s, want in ((HOST, HOST, HOST), (HERE, HOST, HERE), (HOST, HERE, HERE), (HERE, HERE, HERE)):
        where.update({codes.data_ptr(): c, scales.data_ptr(): s})
        assert tb.MxRows(codes, scales).device == want
    where.update({codes.data_ptr(): HERE, scales.data_ptr(): OTHER})
    with pytest.raises(ValueError):
        tb.MxRows(codes, scales)
