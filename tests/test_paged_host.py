"""Host-side checks of a paged cache's entry points: what they refuse, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2503_07518_amd import binding as tb

P = 0x10000  # never dereferenced: every call below fails validation first, or has nothing to do
INV, UNS, WS, OK = tb.TB_ERR_INVALID_ARG, tb.TB_ERR_UNSUPPORTED, tb.TB_ERR_WORKSPACE, tb.TB_OK


@pytest.fixture(scope="module", autouse=True)
def lib():
    return tb.load_library()


def desc(**kw):
    d = tb.tb_cache_desc(2, 8, 2, 128, 32, tb.TB_BF16, 1000, 0, 0, 128, 0, 0, 128, 0, 0, 32)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def cache(**kw):
    c = tb.tb_paged_cache(P, P, P, 200, 16, 64, 64, 2 * 16 * 128, 16 * 128, 128, 2 * 16 * 128, 16 * 128, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(heads=8, **kw):
    r = tb.tb_token_rows(P, heads * 128, 128)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(lib, d=None, c=None, T=4, cu=P, lens=P, f=P, rot=128, q=0, k=0, v=0, qo=0, ko=0):
    q, qo = (rows() if x == 0 else x for x in (q, qo))
    k, v, ko = (rows(2) if x == 0 else x for x in (k, v, ko))
    return lib.tb_append_paged_kv(ref(d or desc()), ref(cache() if c is None else c), T, cu, lens, None, f, rot, 0, ref(q), ref(k), ref(v), ref(qo), ref(ko), None)


def attn(lib, d=None, c=None, T=4, cu=P, lens=P, most=4, q=0, window=0, out=0, ws=P, ws_bytes=1 << 40):
    q, out = (rows() if x == 0 else x for x in (q, out))
    return lib.tb_paged_attn(ref(d or desc()), ref(cache() if c is None else c), T, cu, lens, most, ref(q), window, 0.1, ref(out), None, ws, ws_bytes, None)


def sparse(lib, d=None, c=None, q=P, idx=P, cnt=P, cap=100, most=100, lo=0, hi=0, out=P, ws=P, ws_bytes=1 << 40):
    return lib.tb_sparse_decode_attn_paged(ref(d or desc()), ref(cache() if c is None else c), q, idx, cnt, cap, most, lo, hi, 0.1, out, None, ws, ws_bytes, None)


CACHES = [
    (INV, dict(c=cache(K=None))), (INV, dict(c=cache(V=None))), (INV, dict(c=cache(table=None))), (INV, dict(c=cache(pages=0))),
    (INV, dict(c=cache(pages=-1))), (INV, dict(c=cache(page=0))), (INV, dict(c=cache(page=-16))), (INV, dict(c=cache(table_len=62))),
    (INV, dict(c=cache(table_len=-1))), (INV, dict(c=cache(table_stride=-64))), (INV, dict(c=cache(k_stride_p=-8))), (INV, dict(c=cache(v_stride_n=64))),
    (UNS, dict(c=cache(page=8, table_len=200))), (UNS, dict(c=cache(page=48))), (UNS, dict(c=cache(page=1 << 17))),
    (UNS, dict(c=cache(k_stride_h=1028))), (UNS, dict(c=cache(v_stride_p=4100))), (UNS, dict(c=cache(K=P + 8))), (UNS, dict(c=cache(V=P + 2))),
    (UNS, dict(c=cache(k_stride_n=1 << 25))), (UNS, dict(c=cache(k_stride_n=1 << 60))), (UNS, dict(c=cache(v_stride_n=1 << 59))), (UNS, dict(d=desc(N=(1 << 30) + 1), c=cache(page=65536, table_len=1 << 20))),
    (INV, dict(d=desc(dtype=5))), (INV, dict(d=desc(Hq=7))), (UNS, dict(d=desc(D=96))), (UNS, dict(d=desc(Hq=32))), (INV, dict(d=desc(N=-1))),
    (UNS, dict(d=desc(B=65536))),
]


@pytest.mark.parametrize("call", [append, attn, sparse])
@pytest.mark.parametrize("want,kw", CACHES)
def test_caches_refused(lib, call, want, kw):
    assert call(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (INV, dict(T=-1)), (INV, dict(lens=None)), (INV, dict(cu=None, T=5)), (UNS, dict(T=(1 << 22) + 1)), (INV, dict(k=None)), (INV, dict(v=None)),
    (INV, dict(q=None)), (INV, dict(qo=None)), (INV, dict(rot=-16)), (INV, dict(rot=144)), (UNS, dict(rot=24)), (INV, dict(f=None)),
    (INV, dict(k=rows(2, rows=None))), (UNS, dict(k=rows(2, rows=P + 8))), (UNS, dict(v=rows(2, stride_t=260))), (INV, dict(ko=rows(2, stride_h=64))), (INV, dict(qo=rows(stride_t=64))),
    (INV, dict(ko=rows(2, stride_t=-256))), (UNS, dict(qo=rows(rows=P + 4))),
    (OK, dict(T=0)), (OK, dict(T=0, k=rows(2, rows=None), v=rows(2, rows=None), ko=None)), (OK, dict(T=0, q=None, qo=None, ko=None, rot=0, f=None)), (OK, dict(d=desc(B=0), T=0, cu=None)),
])
def test_append_refusals(lib, want, kw):
    assert append(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (INV, dict(T=-1)), (INV, dict(lens=None)), (INV, dict(cu=None, T=5)), (INV, dict(most=-1)), (INV, dict(window=-1)), (INV, dict(q=None)),
    (INV, dict(out=None)), (INV, dict(out=rows(stride_h=120))), (INV, dict(out=rows(stride_t=64))), (UNS, dict(q=rows(rows=P + 8))), (UNS, dict(out=rows(stride_t=1028))),
    (WS, dict(ws=None)), (WS, dict(ws=P + 8)), (WS, dict(ws_bytes=100)), (OK, dict(T=0)), (OK, dict(T=0, q=rows(rows=None), out=rows(rows=None))), (OK, dict(most=0)),
    (UNS, dict(T=(1 << 22) + 1)), (UNS, dict(T=1 << 22, most=1 << 22, d=desc(Hq=4096, Hkv=4096), ws_bytes=1 << 62)), (OK, dict(d=desc(B=0), T=0)),
    (OK, dict(d=desc(Hq=0, Hkv=0))),
])
def test_attn_refusals(lib, want, kw):
    assert attn(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (INV, dict(q=None)), (INV, dict(idx=None)), (INV, dict(cnt=None)), (INV, dict(out=None)), (INV, dict(most=101)), (INV, dict(most=-1)),
    (INV, dict(lo=5, hi=4)), (INV, dict(hi=1001)), (INV, dict(lo=-1)), (INV, dict(d=desc(N=0))), (UNS, dict(q=P + 8)), (WS, dict(ws=None)),
    (WS, dict(ws_bytes=64)), (UNS, dict(c=cache(pages=1 << 24))), (OK, dict(d=desc(B=0))),
])
def test_sparse_refusals(lib, want, kw):
    assert sparse(lib, **kw) == want


@pytest.mark.parametrize("dtype", [tb.TB_F32, tb.TB_BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_a_workspace_serves_smaller_calls(dtype, D):
    for B, Hq, Hkv in ((1, 8, 1), (3, 32, 8), (64, 8, 8), (300, 8, 2)):
        def of(T, N):
            return tb.tb_workspace_bytes(tb.TB_OP_PAGED_ATTN, desc(B=B, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, N=N), T)
        sizes = [of(T, 100000) for T in (0, 1, 7, 64, 1000, 8192, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] > 0
        sizes = [of(500, N) for N in (0, 1, 300, 5000, 100000, 1 << 24)]
        assert sizes == sorted(sizes)
    assert tb.tb_workspace_bytes(tb.TB_OP_PAGED_ATTN, desc(D=96), 10) == 0 and tb.tb_workspace_bytes(tb.TB_OP_PAGED_ATTN, desc(), -1) == 0


def make_cache(K=(10, 2, 16, 128), dtype=torch.bfloat16, table=(2, 4)):
    return tb.PagedCache(torch.zeros(K, dtype=dtype), torch.zeros(K, dtype=dtype), torch.zeros(table, dtype=torch.int32))


def test_binding_looks_at_shapes_and_types():
    c = make_cache()
    d = tb.make_paged_desc(64, 8, c)
    q, k = torch.zeros((4, 8, 128), dtype=torch.bfloat16), torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    lens, cu, ws = torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8)
    f = torch.zeros(64)
    for bad in (dict(k=k[:, :1]), dict(k=k.float()), dict(q=q[:3]), dict(q_out=None), dict(lens=lens.long()), dict(cu=cu[:2]), dict(inv_freq=f.double()),
                dict(positions=lens), dict(k_out=q), dict(k=k[..., ::2])):
        args = dict(q=q, k=k, v=k, cu=cu, lens=lens, inv_freq=f, q_out=q, k_out=k)
        args.update(bad)
        with pytest.raises((AssertionError, AttributeError, ValueError)):
            tb.tb_append_paged_kv(d, c, **args)
    for bad in (dict(q=q.float()), dict(out=q[:, :4]), dict(lse=torch.zeros(4, 8).double()), dict(lens=lens[:1])):
        args = dict(q=q, cu=cu, lens=lens, max_new=4, sm_scale=1.0, out=q, lse=None, ws=ws)
        args.update(bad)
        with pytest.raises(AssertionError):
            tb.tb_paged_attn(d, c, **args)
    with pytest.raises(AssertionError):
        tb.PagedCache(c.K, c.V, c.table.long())
    with pytest.raises(AssertionError):
        tb.PagedCache(c.K, c.V[:, :1], c.table)
