"""Pools of pages up to the size that attention over lists takes, 64 GiB each of K and V, and those past it.  Host only: nothing is launched,
as the workspace is refused behind the checks of the pool."""
import ctypes

import pytest

from paper_2503_07518_amd import binding as tb

P = 0x10000
MOST = 1 << 36  # bytes


@pytest.fixture(scope="module", autouse=True)
def lib():
    return tb.load_library()


def call(lib, Hkv, D, dtype, page, pages, k, v):
    """k, v: strides (page, head, row) in elements."""
    d = tb.tb_cache_desc(2, Hkv, Hkv, D, 32, dtype, 100, 0, 0, D, 0, 0, D, 0, 0, 32)
    c = tb.tb_paged_cache(P, P, P, pages, page, 100, 100, *k, *v)
    return lib.tb_sparse_decode_attn_paged(ctypes.byref(d), ctypes.byref(c), P, P, P, 10, 10, 0, 0, 1.0, P, None, None, 0, None)


@pytest.mark.parametrize("dtype,elt", [(tb.TB_BF16, 2), (tb.TB_F32, 4)])
@pytest.mark.parametrize("Hkv", [1, 2, 8])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (128, 65536)])
def test_a_pool_of_64_GiB(lib, dtype, elt, Hkv, D, page):
    packed = (Hkv * page * D, page * D, D)
    pages = MOST // (packed[0] * elt)
    assert pages * packed[0] * elt == MOST
    assert call(lib, Hkv, D, dtype, page, pages, packed, packed) == tb.TB_ERR_WORKSPACE
    assert call(lib, Hkv, D, dtype, page, pages + 1, packed, packed) == tb.TB_ERR_UNSUPPORTED
    # each of the two counts, and K and V side by side are twice as far apart
    wide = (2 * packed[0], *packed[1:])
    for k, v in ((wide, packed), (packed, wide), (wide, wide)):
        assert call(lib, Hkv, D, dtype, page, pages // 2, k, v) == tb.TB_ERR_WORKSPACE
        assert call(lib, Hkv, D, dtype, page, pages // 2 + 1, k, v) == tb.TB_ERR_UNSUPPORTED


def test_pools_of_one_page_and_of_large_strides(lib):
    def of(pages, stride_p, stride_n=128):
        return call(lib, 1, 128, tb.TB_BF16, 16, pages, (stride_p, 0, stride_n), (2048, 0, 128))
    assert of(1, 1 << 62) == tb.TB_ERR_WORKSPACE  # (nothing lies a page further on)
    for pages in (2, 3, 1000, (1 << 31) - 1):
        assert of(pages, 1 << 62) == of(pages, (1 << 63) - 8) == tb.TB_ERR_UNSUPPORTED
    # the last row of two pages ends with the 64 GiB, or 16 bytes behind them
    most = MOST // 2 - 128
    assert of(2, most - 15 * 128) == tb.TB_ERR_WORKSPACE and of(2, most - 15 * 128 + 8) == tb.TB_ERR_UNSUPPORTED
    assert of(2, most - 15 * 4096, 4096) == tb.TB_ERR_WORKSPACE and of(2, most - 15 * 4096 + 8, 4096) == tb.TB_ERR_UNSUPPORTED
