"""ctypes binding of libtokenbutler.so: argument marshalling only.

Every function has the name of the C entry point it calls (``include/tokenbutler.h``) and
passes device pointers of torch tensors plus the current HIP stream.  No step of the path is
computed here; if the HIP library is missing or does not load, importing the ops fails loudly
(there is no fallback).
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtokenbutler.so")

TB_OK, TB_ERR_INVALID_ARG, TB_ERR_UNSUPPORTED, TB_ERR_WORKSPACE, TB_ERR_HIP = 0, 1, 2, 3, 4
TB_F32, TB_BF16 = 0, 1
TB_OP_SELECT, TB_OP_ATTN, TB_OP_DECODE_STEP, TB_OP_ATTN_MX, TB_OP_PAGED_ATTN = 1, 2, 3, 4, 5
MX_BLOCK = 32  # elements that share a scale in a 4-bit cache

EXPORTS = (
    "tb_project_keys", "tb_score", "tb_select_topk", "tb_expand_neighbors", "tb_sparse_decode_attn",
    "tb_sparse_decode_attn_shared", "tb_sparse_decode_attn_static",
    "tb_gather_kv", "tb_gather_important", "tb_append_kv", "tb_buffered_decode_attn", "tb_append_buffered_decode_attn", "tb_migrate_buffered_decode_attn", "tb_predict_queries", "tb_decode_step",
    "tb_quantize_mx", "tb_dequantize_mx", "tb_score_mx", "tb_sparse_decode_attn_mx", "tb_sparse_decode_attn_shared_mx",
    "tb_append_paged_kv", "tb_paged_attn", "tb_sparse_decode_attn_paged",
    "tb_workspace_bytes", "tb_workspace_init", "tb_read_stream_probe", "tb_status_string", "tb_version",
)


class TbError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {status_string(code)} (tb_status {code})")


class tb_cache_desc(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
        ("Dimp", ctypes.c_int32), ("dtype", ctypes.c_int32), ("N", ctypes.c_int64),
        ("k_stride_b", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_n", ctypes.c_int64),
        ("v_stride_b", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_n", ctypes.c_int64),
        ("ki_stride_b", ctypes.c_int64), ("ki_stride_h", ctypes.c_int64), ("ki_stride_n", ctypes.c_int64),
    ]


class tb_mx_rows(ctypes.Structure):
    _fields_ = [
        ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("N", ctypes.c_int64),
        ("code_stride_b", ctypes.c_int64), ("code_stride_h", ctypes.c_int64), ("code_stride_n", ctypes.c_int64),
        ("scale_stride_b", ctypes.c_int64), ("scale_stride_h", ctypes.c_int64), ("scale_stride_n", ctypes.c_int64),
    ]


class tb_paged_cache(ctypes.Structure):
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("table", ctypes.c_void_p),
        ("pages", ctypes.c_int32), ("page", ctypes.c_int32), ("table_len", ctypes.c_int32), ("table_stride", ctypes.c_int64),
        ("k_stride_p", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_n", ctypes.c_int64),
        ("v_stride_p", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_n", ctypes.c_int64),
    ]


class tb_token_rows(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_void_p), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class tb_predictor_desc(ctypes.Structure):
    _fields_ = [
        ("E", ctypes.c_int32), ("hidden", ctypes.c_int32), ("G", ctypes.c_int32), ("Hq", ctypes.c_int32),
        ("Dimp", ctypes.c_int32), ("dtype", ctypes.c_int32), ("ln_eps", ctypes.c_float),
    ]


_lib: Optional[ctypes.CDLL] = None


def load_library() -> ctypes.CDLL:
    """Load libtokenbutler.so from the package directory.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2503_07518_amd.build` "
            "(hipcc, --offload-arch=gfx950).  There is no fallback implementation.")
    L = ctypes.CDLL(LIB_PATH)
    i32, i64, f32, vp, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    dp = ctypes.POINTER(tb_cache_desc)
    L.tb_project_keys.argtypes = [dp, vp, vp, i32, vp, i64, i64, vp]
    L.tb_score.argtypes = [dp, vp, vp, f32, vp, i64, vp]
    L.tb_select_topk.argtypes = [dp, vp, i64, i32, i32, i32, vp, vp, i64, vp, sz, vp]
    L.tb_expand_neighbors.argtypes = [i32, i32, i64, i32, i32, vp, vp, i64, vp, vp, i64, vp]
    L.tb_sparse_decode_attn.argtypes = [dp, vp, vp, vp, vp, vp, i64, i64, i64, i64, f32, vp, vp, vp, sz, vp]
    L.tb_sparse_decode_attn_shared.argtypes = L.tb_sparse_decode_attn.argtypes
    L.tb_sparse_decode_attn_static.argtypes = [dp, vp, vp, vp, vp, vp, i64, i64, i64, i64, f32, vp, vp, vp]
    L.tb_decode_step.argtypes = [dp, vp, vp, f32, vp, vp, vp, i32, i32, i32, f32, vp, i64, vp, vp, i64, vp, vp,
                                 vp, sz, vp]
    L.tb_gather_kv.argtypes = [dp, vp, vp, vp, vp, i64, i64, vp, vp, i64, vp]
    L.tb_gather_important.argtypes = [dp, vp, vp, vp, vp, i64, i64, i32, i32, vp, vp, i64, vp, vp]
    L.tb_append_kv.argtypes = [dp, vp, vp, i64, dp, vp, vp, i64, i64, vp]
    L.tb_buffered_decode_attn.argtypes = [dp, vp, vp, vp, i64, vp, i64, vp, vp, i64, i64, f32, vp, vp, vp, sz, vp]
    L.tb_append_buffered_decode_attn.argtypes = [dp, vp, vp, i64, dp, vp, vp, vp, i64, vp, i64, vp, vp, i64, i64, i64, f32, vp, vp, vp, sz, vp]
    L.tb_migrate_buffered_decode_attn.argtypes = [dp, vp, vp, vp, vp, i64, i64, i32, i32, vp, i64, dp, vp, vp, vp, i64, vp, vp, i64, i64, i64, f32, vp, vp, vp,
                                                  sz, vp]
    L.tb_predict_queries.argtypes = [ctypes.POINTER(tb_predictor_desc), i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    mp = ctypes.POINTER(tb_mx_rows)
    L.tb_quantize_mx.argtypes = [dp, vp, vp, vp, i64, mp, mp, mp, i64, i64, vp]
    L.tb_dequantize_mx.argtypes = [dp, mp, mp, mp, i64, vp, vp, vp, i64, i64, vp]
    L.tb_score_mx.argtypes = [dp, vp, mp, f32, vp, i64, vp]
    L.tb_sparse_decode_attn_mx.argtypes = [dp, vp, mp, mp, vp, vp, i64, i64, i64, i64, f32, vp, vp, vp, sz, vp]
    L.tb_sparse_decode_attn_shared_mx.argtypes = L.tb_sparse_decode_attn_mx.argtypes
    pp, rp = ctypes.POINTER(tb_paged_cache), vp  # (rp: tb_token_rows by their address)
    L.tb_append_paged_kv.argtypes = [dp, pp, i64, vp, vp, vp, vp, i32, i32, rp, rp, rp, rp, rp, vp]
    L.tb_paged_attn.argtypes = [dp, pp, i64, vp, vp, i64, rp, i64, f32, rp, vp, vp, sz, vp]
    L.tb_sparse_decode_attn_paged.argtypes = [dp, pp, vp, vp, vp, i64, i64, i64, i64, f32, vp, vp, vp, sz, vp]
    L.tb_workspace_bytes.argtypes = [i32, dp, i64]
    L.tb_workspace_bytes.restype = sz
    L.tb_workspace_init.argtypes = [vp, sz, vp]
    L.tb_read_stream_probe.argtypes = [vp, sz, vp, vp]
    L.tb_status_string.argtypes = [ctypes.c_int]
    L.tb_status_string.restype = ctypes.c_char_p
    L.tb_version.restype = i32
    for name in EXPORTS:
        if name not in ("tb_workspace_bytes", "tb_status_string", "tb_version"):
            getattr(L, name).restype = ctypes.c_int
    global _several_devices
    _several_devices = torch.cuda.device_count() != 1
    _lib = L
    return L


def status_string(code: int) -> str:
    return load_library().tb_status_string(int(code)).decode()


def _check(code: int, what: str) -> None:
    if code != TB_OK:
        raise TbError(code, what)


# (plain integers: the argument types turn them into pointers, at a third of the cost of c_void_p objects)
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# the current stream's handle without a Stream object around it, which cost 3 us a call: more than the rest of one (torch
# does not promise this function: without it the object serves)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_several_devices = True  # (set when the library is loaded: with one GPU no tensor is on another, and up to 0.8 us a call are saved)


def _stream_on(device: int, stream=None, also=()) -> int:
    """The handle of `stream`, or of the current one, for tensors on GPU number `device` (-1: in host memory) and those in `also` (None:
    left out).  The kernels run on the current device: tensors on another one are refused."""
    current = _get_device()
    if device != current and device >= 0:
        raise ValueError(f"tensors on cuda:{device}, and cuda:{current} is the current device")
    for t in also:
        if t is not None:
            device = t.get_device()
            if device != current and device >= 0:
                raise ValueError(f"tensors on cuda:{device}, and cuda:{current} is the current device")
    if stream is not None:
        return stream.cuda_stream
    return _stream() if _raw_stream is None else _raw_stream(current)


def _dtype_code(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return TB_F32
    if dtype == torch.bfloat16:
        return TB_BF16
    raise TypeError(f"unsupported element type {dtype}")


def _strides3(t: torch.Tensor) -> Tuple[int, int, int]:
    st = t.stride()
    assert len(st) == 4 and st[3] == 1, "cache tensors are [B, Hkv, N, D] with D contiguous"
    return st[:3]


def make_desc(N: int, Hq: int, K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None,
              Kimp: Optional[torch.Tensor] = None, D: Optional[int] = None, Dimp: Optional[int] = None) -> tb_cache_desc:
    """Describe one layer's cache from the tensors at hand.  Missing tensors get neutral
    strides; D / Dimp may be given explicitly when the tensor that carries them is absent."""
    if K is not None:
        k = _strides3(K)
        B, Hkv, _, inner = K.shape
        dtype = K.dtype
    else:
        ref = Kimp if Kimp is not None else V
        assert ref is not None
        B, Hkv = ref.shape[0], ref.shape[1]
        inner = 128 if V is None else V.shape[3]
        k = None
        dtype = ref.dtype
    if D is None:
        D = inner
    k = k or (0, 0, D)
    v = k if V is None else _strides3(V)
    if Kimp is not None:
        if Dimp is None:
            Dimp = Kimp.shape[3]
        ki = _strides3(Kimp)
    else:
        if Dimp is None:
            Dimp = 32
        ki = (0, 0, Dimp)
    return tb_cache_desc(B, Hq, Hkv, D, Dimp, _dtype_code(dtype), N, *k, *v, *ki)


class MxRows:
    """Rows in microscaled 4-bit floating point: codes uint8 [B, Hkv, N, inner / 2], scales uint8 [B, Hkv, N, inner / 32]."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        assert codes.dtype == scales.dtype == torch.uint8
        assert codes.shape[:3] == scales.shape[:3] and codes.shape[3] * 2 == scales.shape[3] * MX_BLOCK
        self.codes, self.scales = codes, scales
        self.desc = tb_mx_rows(codes.data_ptr(), scales.data_ptr(), codes.shape[2], *_strides3(codes), *_strides3(scales))
        self.ref = ctypes.byref(self.desc)
        on = (codes.get_device(), scales.get_device())
        self.device = max(on)
        if -1 not in on and on[0] != on[1]:
            raise ValueError(f"codes on cuda:{on[0]}, scales on cuda:{on[1]}")

    def get_device(self) -> int:
        """The GPU that the rows are on (-1: in host memory)."""
        return self.device

    @property
    def inner(self) -> int:
        return self.codes.shape[3] * 2


class MxCache:
    """A layer's cache in microscaled 4-bit floating point, for Ncap tokens: K and V of a token side by side (a line of 128 bytes at
    D = 128), and the projected keys (Dimp = 0: none)."""

    def __init__(self, B: int, Hkv: int, Ncap: int, D: int, Dimp: int = 0, device="cuda"):
        codes = torch.zeros((B, Hkv, Ncap, 2, D // 2), dtype=torch.uint8, device=device)
        scales = torch.zeros((B, Hkv, Ncap, 2, D // MX_BLOCK), dtype=torch.uint8, device=device)
        self.K, self.V = (MxRows(codes[:, :, :, t], scales[:, :, :, t]) for t in (0, 1))
        self.Kimp = None
        if Dimp:
            self.Kimp = MxRows(torch.zeros((B, Hkv, Ncap, Dimp // 2), dtype=torch.uint8, device=device),
                               torch.zeros((B, Hkv, Ncap, Dimp // MX_BLOCK), dtype=torch.uint8, device=device))


def make_mx_desc(N: int, Hq: int, dtype: torch.dtype, K: Optional[MxRows] = None, Kimp: Optional[MxRows] = None) -> tb_cache_desc:
    """Describe a layer whose rows are in 4 bits: its shape, and the element type of the queries."""
    ref = K if K is not None else Kimp
    B, Hkv = ref.codes.shape[:2]
    D, Dimp = 128 if K is None else K.inner, 32 if Kimp is None else Kimp.inner
    return tb_cache_desc(B, Hq, Hkv, D, Dimp, _dtype_code(dtype), N, 0, 0, D, 0, 0, D, 0, 0, Dimp)


class PagedCache:
    """A layer's cache in pages: K, V [pages, Hkv, page, D], table int32 [B, entries]; row n of sequence b is row n % page of page
    table[b, n // page].  The tensors stay the caller's: pages are handed out by writing into the table."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, table: torch.Tensor):
        assert K.shape == V.shape and K.dtype == V.dtype and table.dtype == torch.int32 and table.dim() == 2
        assert table.shape[1] < 2 or table.stride(1) == 1
        self.K, self.V, self.table = K, V, table
        self.desc = tb_paged_cache(K.data_ptr(), V.data_ptr(), table.data_ptr(), K.shape[0], K.shape[2], table.shape[1],
                                   table.stride(0) if table.shape[0] > 1 else table.shape[1], *_strides3(K), *_strides3(V))
        self.ref = ctypes.byref(self.desc)
        self.device, self.dtype, self.B = K.get_device(), K.dtype, table.shape[0]
        if not self.device == V.get_device() == table.get_device():
            raise ValueError(f"K on {K.device}, V on {V.device}, table on {table.device}")

    def get_device(self) -> int:
        """The GPU that the pages are on (-1: in host memory)."""
        return self.device


def make_paged_desc(N: int, Hq: int, cache: PagedCache) -> tb_cache_desc:
    """Describe a layer whose cache is in pages; N: the most rows that a sequence has."""
    _, Hkv, _, D = cache.K.shape
    return tb_cache_desc(cache.table.shape[0], Hq, Hkv, D, 32, _dtype_code(cache.K.dtype), N, 0, 0, D, 0, 0, D, 0, 0, 32)


# tb_token_rows of a call's tensors, one after the other: a fifth of the cost of a structure each
_two_rows, _five_rows = ctypes.c_int64 * 6, ctypes.c_int64 * 15
_pack_two, _pack_five = struct.Struct("6q").pack, struct.Struct("15q").pack
_ROWS = ctypes.sizeof(tb_token_rows)


def tb_version() -> int:
    return int(load_library().tb_version())


def tb_workspace_bytes(op: int, desc: tb_cache_desc, max_count: int = 0) -> int:
    return int(load_library().tb_workspace_bytes(op, ctypes.byref(desc), int(max_count)))


def tb_workspace_init(ws: torch.Tensor, stream=None) -> None:
    _check(load_library().tb_workspace_init(_ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "tb_workspace_init")


def tb_read_stream_probe(src: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """Read `src` once with a plain streaming kernel (a bandwidth calibration, see the header)."""
    _check(load_library().tb_read_stream_probe(_ptr(src), src.numel() * src.element_size(), _ptr(sink),
                                               _stream(stream)), "tb_read_stream_probe")


def new_workspace(op: int, desc: tb_cache_desc, max_count: int = 0, device="cuda") -> torch.Tensor:
    """Allocate (torch, device memory) and zero a workspace for `op`."""
    nbytes = tb_workspace_bytes(op, desc, max_count)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    tb_workspace_init(ws)
    return ws


def tb_project_keys(desc, K, W, Kimp, n_begin: int, n_end: int, stream=None) -> None:
    Hw = W.shape[0]
    assert W.is_contiguous()
    _check(load_library().tb_project_keys(ctypes.byref(desc), _ptr(K), _ptr(W), Hw, _ptr(Kimp), n_begin, n_end,
                                          _stream(stream)), "tb_project_keys")


def tb_score(desc, q_imp, Kimp, scale: float, scores, stream=None) -> None:
    assert q_imp.is_contiguous() and scores.stride(-1) == 1
    _check(load_library().tb_score(ctypes.byref(desc), _ptr(q_imp), _ptr(Kimp), scale, _ptr(scores),
                                   scores.stride(-2), _stream(stream)), "tb_score")


def tb_select_topk(desc, scores, k: int, sink: int, window: int, idx, count, ws, stream=None) -> None:
    _check(load_library().tb_select_topk(ctypes.byref(desc), _ptr(scores), scores.stride(-2), k, sink, window,
                                         _ptr(idx), _ptr(count), idx.stride(-2), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream(stream)), "tb_select_topk")


def tb_gather_kv(desc, K, V, idx, count, max_count: int, Kbuf, Vbuf, stream=None) -> None:
    assert Kbuf.is_contiguous() and Vbuf.is_contiguous() and Kbuf.shape == Vbuf.shape
    _check(load_library().tb_gather_kv(ctypes.byref(desc), _ptr(K), _ptr(V), _ptr(idx), _ptr(count), idx.stride(-2),
                                       max_count, _ptr(Kbuf), _ptr(Vbuf), Kbuf.shape[2], _stream(stream)),
           "tb_gather_kv")


def tb_gather_important(desc, K, V, idx, count, max_count: int, skip_front: int, skip_back: int, Kbuf, Vbuf,
                        count_out, stream=None) -> None:
    assert Kbuf.is_contiguous() and Vbuf.is_contiguous() and Kbuf.shape == Vbuf.shape
    _check(load_library().tb_gather_important(ctypes.byref(desc), _ptr(K), _ptr(V), _ptr(idx), _ptr(count),
                                              idx.stride(-2), max_count, skip_front, skip_back, _ptr(Kbuf), _ptr(Vbuf),
                                              Kbuf.shape[2], _ptr(count_out), _stream(stream)), "tb_gather_important")


def tb_append_kv(src, K, V, src_row: int, dst, Kdst, Vdst, dst_row: int, rows: int = 1, stream=None) -> None:
    """Kdst/Vdst[b, h, dst_row + i] = K/V[b, h, src_row + i] for i < rows, every KV head of the batch."""
    _check(load_library().tb_append_kv(ctypes.byref(src), _ptr(K), _ptr(V), src_row, ctypes.byref(dst), _ptr(Kdst), _ptr(Vdst), dst_row,
                                       rows, _stream(stream)), "tb_append_kv")


def tb_buffered_decode_attn(desc, q, Kbuf, Vbuf, count, max_count: int, K, V, sm_scale: float, out, lse, ws,
                            tail_begin: int = 0, tail_end: int = 0, stream=None) -> None:
    assert Kbuf.is_contiguous() and Vbuf.is_contiguous() and Kbuf.shape == Vbuf.shape
    _check(load_library().tb_buffered_decode_attn(ctypes.byref(desc), _ptr(q), _ptr(Kbuf), _ptr(Vbuf), Kbuf.shape[2],
                                                  _ptr(count), max_count, _ptr(K), _ptr(V), tail_begin, tail_end,
                                                  sm_scale, _ptr(out), _ptr(lse), _ptr(ws),
                                                  ws.numel() * ws.element_size(), _stream(stream)),
           "tb_buffered_decode_attn")


def tb_append_buffered_decode_attn(src, K_src, V_src, src_row: int, desc, q, Kbuf, Vbuf, count, max_count: int, K, V, dst_row: int,
                                   sm_scale: float, out, lse, ws, tail_begin: int = 0, tail_end: int = 0, stream=None) -> None:
    """tb_append_kv of one row into row dst_row of the cache K, V, and tb_buffered_decode_attn over it, in one launch."""
    assert Kbuf.is_contiguous() and Vbuf.is_contiguous() and Kbuf.shape == Vbuf.shape
    _check(load_library().tb_append_buffered_decode_attn(ctypes.byref(src), _ptr(K_src), _ptr(V_src), src_row, ctypes.byref(desc), _ptr(q),
                                                         _ptr(Kbuf), _ptr(Vbuf), Kbuf.shape[2], _ptr(count), max_count, _ptr(K), _ptr(V),
                                                         dst_row, tail_begin, tail_end, sm_scale, _ptr(out), _ptr(lse), _ptr(ws),
                                                         ws.numel() * ws.element_size(), _stream(stream)),
           "tb_append_buffered_decode_attn")


def tb_migrate_buffered_decode_attn(src, K_src, V_src, idx, count, max_count: int, skip_front: int, skip_back: int, count_out, src_row: int, desc, q,
                                    Kbuf, Vbuf, K, V, dst_row: int, sm_scale: float, out, lse, ws, tail_begin: int = 0, tail_end: int = 0,
                                    stream=None) -> None:
    """tb_gather_important of the lists into the buffers, (src_row >= 0) tb_append_kv of one row into row dst_row of the cache K, V, and
    tb_buffered_decode_attn over both, in one launch."""
    assert Kbuf.is_contiguous() and Vbuf.is_contiguous() and Kbuf.shape == Vbuf.shape
    _check(load_library().tb_migrate_buffered_decode_attn(
        ctypes.byref(src), _ptr(K_src), _ptr(V_src), _ptr(idx), _ptr(count), idx.stride(-2), max_count, skip_front, skip_back, _ptr(count_out), src_row,
        ctypes.byref(desc), _ptr(q), _ptr(Kbuf), _ptr(Vbuf), Kbuf.shape[2], _ptr(K), _ptr(V), dst_row, tail_begin, tail_end, sm_scale, _ptr(out),
        _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "tb_migrate_buffered_decode_attn")


def tb_predict_queries(h, gamma, beta, W1, b1, W2, b2, G: int, Hq: int, Dimp: int, hidden_act, ln_act, q_imp,
                       ln_eps: float = 1e-5, stream=None) -> None:
    """q_imp[G][B][Hq][Dimp] = MLP(LN(h)); W1 [hidden][E], W2 [G*Hq*Dimp][hidden] (torch Linear layout)."""
    B, E = h.shape
    hidden = W1.shape[0]
    for t in (h, gamma, beta, W1, b1, W2, b2, hidden_act, ln_act, q_imp):
        assert t.is_contiguous()
    assert W1.shape == (hidden, E) and W2.shape == (G * Hq * Dimp, hidden)
    assert hidden_act.dtype == torch.float32 and hidden_act.shape == (B, hidden)
    assert ln_act.dtype == torch.float32 and ln_act.shape == (B, E)
    assert q_imp.shape == (G, B, Hq, Dimp) and q_imp.dtype == h.dtype
    p = tb_predictor_desc(E, hidden, G, Hq, Dimp, _dtype_code(h.dtype), ln_eps)
    _check(load_library().tb_predict_queries(ctypes.byref(p), B, _ptr(h), _ptr(gamma), _ptr(beta), _ptr(W1), _ptr(b1),
                                             _ptr(W2), _ptr(b2), _ptr(hidden_act), _ptr(ln_act), _ptr(q_imp), _stream(stream)),
           "tb_predict_queries")


def tb_expand_neighbors(B: int, Hq: int, N: int, radius: int, mode: int, idx_in, count_in, idx_out, count_out,
                        stream=None) -> None:
    _check(load_library().tb_expand_neighbors(B, Hq, N, radius, mode, _ptr(idx_in), _ptr(count_in),
                                              idx_in.stride(-2), _ptr(idx_out), _ptr(count_out), idx_out.stride(-2),
                                              _stream(stream)), "tb_expand_neighbors")


def tb_sparse_decode_attn(desc, q, K, V, idx, count, max_count: int, sm_scale: float, out, lse, ws,
                          tail_begin: int = 0, tail_end: int = 0, stream=None) -> None:
    assert q.is_contiguous() and out.is_contiguous()
    _check(load_library().tb_sparse_decode_attn(ctypes.byref(desc), _ptr(q), _ptr(K), _ptr(V), _ptr(idx),
                                                _ptr(count), idx.stride(-2), max_count, tail_begin, tail_end,
                                                sm_scale, _ptr(out), _ptr(lse), _ptr(ws),
                                                ws.numel() * ws.element_size(), _stream(stream)),
           "tb_sparse_decode_attn")


def tb_sparse_decode_attn_static(desc, q, K, V, idx, count, max_count: int, sm_scale: float, out, lse,
                                 tail_begin: int = 0, tail_end: int = 0, stream=None) -> None:
    """tb_sparse_decode_attn with the library's own scratch (no workspace, no allocation)."""
    assert q.is_contiguous() and out.is_contiguous()
    _check(load_library().tb_sparse_decode_attn_static(ctypes.byref(desc), _ptr(q), _ptr(K), _ptr(V), _ptr(idx),
                                                       _ptr(count), idx.stride(-2), max_count, tail_begin,
                                                       tail_end, sm_scale, _ptr(out), _ptr(lse), _stream(stream)),
           "tb_sparse_decode_attn_static")


def tb_sparse_decode_attn_shared(desc, q, K, V, idx, count, max_count: int, sm_scale: float, out, lse, ws,
                                 tail_begin: int = 0, tail_end: int = 0, stream=None) -> None:
    """idx: int32 [B][idx_cap] (or [B][1][idx_cap]), count: int32 [B]; one list for all heads."""
    assert q.is_contiguous() and out.is_contiguous()
    _check(load_library().tb_sparse_decode_attn_shared(ctypes.byref(desc), _ptr(q), _ptr(K), _ptr(V), _ptr(idx),
                                                       _ptr(count), idx.stride(-2), max_count, tail_begin,
                                                       tail_end, sm_scale, _ptr(out), _ptr(lse), _ptr(ws),
                                                       ws.numel() * ws.element_size(), _stream(stream)),
           "tb_sparse_decode_attn_shared")


def tb_decode_step(desc, q_imp, Kimp, score_scale: float, q, K, V, k: int, sink: int, window: int, sm_scale: float,
                   scores, idx, count, out, lse, ws, stream=None) -> None:
    assert q.is_contiguous() and q_imp.is_contiguous() and out.is_contiguous()
    _check(load_library().tb_decode_step(ctypes.byref(desc), _ptr(q_imp), _ptr(Kimp), score_scale, _ptr(q), _ptr(K),
                                         _ptr(V), k, sink, window, sm_scale, _ptr(scores), scores.stride(-2),
                                         _ptr(idx), _ptr(count), idx.stride(-2), _ptr(out), _ptr(lse), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream(stream)), "tb_decode_step")


# (The calls of the 4-bit cache spell their arguments out: a function around every pointer costs 0.4 us of a call's 5.5.)
def tb_quantize_mx(desc, K, V, Kimp, src_row: int, Kq: Optional[MxRows], Vq: Optional[MxRows], Kimpq: Optional[MxRows], dst_row: int,
                   rows: int, stream=None) -> None:
    """Rows src_row + i of K, V and Kimp (desc; None: left out) to rows dst_row + i of Kq, Vq and Kimpq, i < rows."""
    to = Kq or Vq or Kimpq
    rc = (_lib or load_library()).tb_quantize_mx(
        ctypes.byref(desc), None if K is None else K.data_ptr(), None if V is None else V.data_ptr(),
        None if Kimp is None else Kimp.data_ptr(), src_row, None if Kq is None else Kq.ref, None if Vq is None else Vq.ref,
        None if Kimpq is None else Kimpq.ref, dst_row, rows, _stream_on(
            -1 if to is None else to.device, stream, (K, V, Kimp, Vq, Kimpq) if _several_devices else ()))
    if rc:
        _check(rc, "tb_quantize_mx")


def tb_dequantize_mx(desc, Kq: Optional[MxRows], Vq: Optional[MxRows], Kimpq: Optional[MxRows], src_row: int, K, V, Kimp, dst_row: int,
                     rows: int, stream=None) -> None:
    """The values that rows src_row + i of Kq, Vq and Kimpq stand for to rows dst_row + i of K, V and Kimp (desc), i < rows."""
    rows_of = Kq or Vq or Kimpq
    rc = (_lib or load_library()).tb_dequantize_mx(
        ctypes.byref(desc), None if Kq is None else Kq.ref, None if Vq is None else Vq.ref, None if Kimpq is None else Kimpq.ref, src_row,
        None if K is None else K.data_ptr(), None if V is None else V.data_ptr(), None if Kimp is None else Kimp.data_ptr(), dst_row, rows,
        _stream_on(-1 if rows_of is None else rows_of.device, stream, (K, V, Kimp, Vq, Kimpq) if _several_devices else ()))
    if rc:
        _check(rc, "tb_dequantize_mx")


def tb_score_mx(desc, q_imp, Kimp: MxRows, scale: float, scores, stream=None) -> None:
    assert q_imp.is_contiguous() and scores.stride(-1) == 1
    rc = (_lib or load_library()).tb_score_mx(ctypes.byref(desc), q_imp.data_ptr(), Kimp.ref, scale, scores.data_ptr(), scores.stride(-2),
                                              _stream_on(scores.get_device(), stream, (q_imp, Kimp) if _several_devices else ()))
    if rc:
        _check(rc, "tb_score_mx")


def tb_sparse_decode_attn_mx(desc, q, K: MxRows, V: MxRows, idx, count, max_count: int, sm_scale: float, out, lse, ws, tail_begin: int = 0,
                             tail_end: int = 0, stream=None) -> None:
    """idx and count may be None with max_count = 0: the dense range alone."""
    assert q.is_contiguous() and out.is_contiguous()
    rc = (_lib or load_library()).tb_sparse_decode_attn_mx(
        ctypes.byref(desc), q.data_ptr(), K.ref, V.ref, None if idx is None else idx.data_ptr(), None if count is None else count.data_ptr(),
        0 if idx is None else idx.stride(-2), max_count, tail_begin, tail_end, sm_scale, out.data_ptr(), None if lse is None else lse.data_ptr(),
        ws.data_ptr(), ws.nbytes, _stream_on(out.get_device(), stream, (q, K, V, idx, count, lse, ws) if _several_devices else ()))
    if rc:
        _check(rc, "tb_sparse_decode_attn_mx")


def tb_sparse_decode_attn_shared_mx(desc, q, K: MxRows, V: MxRows, idx, count, max_count: int, sm_scale: float, out, lse, ws,
                                    tail_begin: int = 0, tail_end: int = 0, stream=None) -> None:
    """idx: int32 [B][idx_cap] (or [B][1][idx_cap]), count: int32 [B]; one list for all heads."""
    assert q.is_contiguous() and out.is_contiguous()
    rc = (_lib or load_library()).tb_sparse_decode_attn_shared_mx(
        ctypes.byref(desc), q.data_ptr(), K.ref, V.ref, None if idx is None else idx.data_ptr(), None if count is None else count.data_ptr(),
        0 if idx is None else idx.stride(-2), max_count, tail_begin, tail_end, sm_scale, out.data_ptr(), None if lse is None else lse.data_ptr(),
        ws.data_ptr(), ws.nbytes, _stream_on(out.get_device(), stream, (q, K, V, idx, count, lse, ws) if _several_devices else ()))
    if rc:
        _check(rc, "tb_sparse_decode_attn_shared_mx")


def _check_tokens(desc, cache: PagedCache, cu, lens) -> None:
    B = cache.B
    assert desc.B == B and lens.dtype is torch.int32 and lens.shape == (B,) and lens.is_contiguous()
    assert cu is None or (cu.dtype is torch.int32 and cu.shape == (B + 1,) and cu.is_contiguous())


# (The calls below spell their arguments out, as those of the 4-bit cache do, and look at each tensor's shape and strides once: 10 us of
# host time for the first one otherwise, now 6.)
def tb_append_paged_kv(desc, cache: PagedCache, q, k, v, cu, lens, inv_freq, q_out=None, k_out=None, positions=None,
                       interleaved: bool = False, stream=None) -> None:
    """Rows of the new tokens k, v [T, Hkv, D] into the cache, k (also to k_out) and q [T, Hq, D] (to q_out; both may be None) rotated by
    positions[t] * inv_freq[i] (int32 [T], None: the token's row; fp32 [rot / 2], None: no rotation).  cu: int32 [B + 1], None: as many
    tokens of every sequence; lens: int32 [B], the rows of the sequences with the new tokens."""
    shape, dtype = k.shape, cache.dtype
    T, Hkv, D = shape
    k_t, k_h, k_d = k.stride()
    v_t, v_h, v_d = v.stride()
    assert v.shape == shape and Hkv == desc.Hkv and D == desc.D and k.dtype is dtype and v.dtype is dtype and k_d == v_d == 1
    qp = qop = kop = 0
    q_t = q_h = qo_t = qo_h = ko_t = ko_h = 0
    if q is not None or q_out is not None:
        q_t, q_h, q_d = q.stride()
        qo_t, qo_h, qo_d = q_out.stride()
        assert q.shape == q_out.shape == (T, desc.Hq, D) and q.dtype is dtype and q_out.dtype is dtype and q_d == qo_d == 1
        qp, qop = q.data_ptr(), q_out.data_ptr()
    if k_out is not None:
        ko_t, ko_h, ko_d = k_out.stride()
        assert k_out.shape == shape and k_out.dtype is dtype and ko_d == 1
        kop = k_out.data_ptr()
    rot, fp = 0, None
    if inv_freq is not None:
        (rot,) = inv_freq.shape
        assert inv_freq.dtype is torch.float32 and (rot < 2 or inv_freq.stride(0) == 1)
        rot, fp = 2 * rot, inv_freq.data_ptr()
    assert positions is None or (positions.dtype is torch.int32 and positions.is_contiguous() and positions.shape == (T,))
    _check_tokens(desc, cache, cu, lens)
    rows = _five_rows.from_buffer_copy(_pack_five(qp, q_t, q_h, k.data_ptr(), k_t, k_h, v.data_ptr(), v_t, v_h, qop, qo_t, qo_h, kop, ko_t, ko_h))
    at = ctypes.addressof(rows)
    rc = (_lib or load_library()).tb_append_paged_kv(
        ctypes.byref(desc), cache.ref, T, None if cu is None else cu.data_ptr(), lens.data_ptr(), None if positions is None else positions.data_ptr(), fp,
        rot, interleaved, None if q is None else at, at + _ROWS, at + 2 * _ROWS, None if q is None else at + 3 * _ROWS,
        None if k_out is None else at + 4 * _ROWS,
        _stream_on(cache.device, stream, (q, k, v, cu, lens, inv_freq, q_out, k_out, positions) if _several_devices else ()))
    if rc:
        _check(rc, "tb_append_paged_kv")


def tb_paged_attn(desc, cache: PagedCache, q, cu, lens, max_new: int, sm_scale: float, out, lse, ws, window: int = 0, stream=None) -> None:
    """Causal attention of the new tokens q [T, Hq, D] over their sequences' rows (their own have been appended), to the last `window` of
    them unless that is 0.  cu and lens as for tb_append_paged_kv; max_new: the most new tokens of a sequence; out: as q; lse: fp32 [T, Hq]
    or None."""
    shape, dtype = q.shape, cache.dtype
    T, Hq, D = shape
    q_t, q_h, q_d = q.stride()
    o_t, o_h, o_d = out.stride()
    assert out.shape == shape and Hq == desc.Hq and D == desc.D and q.dtype is dtype and out.dtype is dtype and q_d == o_d == 1
    assert lse is None or (lse.dtype is torch.float32 and lse.shape == (T, Hq) and lse.is_contiguous())
    _check_tokens(desc, cache, cu, lens)
    rows = _two_rows.from_buffer_copy(_pack_two(q.data_ptr(), q_t, q_h, out.data_ptr(), o_t, o_h))
    at = ctypes.addressof(rows)
    rc = (_lib or load_library()).tb_paged_attn(
        ctypes.byref(desc), cache.ref, T, None if cu is None else cu.data_ptr(), lens.data_ptr(), max_new, at, window, sm_scale, at + _ROWS,
        None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.nbytes,
        _stream_on(cache.device, stream, (q, cu, lens, out, lse, ws) if _several_devices else ()))
    if rc:
        _check(rc, "tb_paged_attn")


def tb_sparse_decode_attn_paged(desc, cache: PagedCache, q, idx, count, max_count: int, sm_scale: float, out, lse, ws, tail_begin: int = 0,
                                tail_end: int = 0, stream=None) -> None:
    """tb_sparse_decode_attn over a cache in pages.  idx: int32 [B, Hq, entries], one list after the other; count: int32 [B, Hq]; out, lse:
    fp32."""
    heads = (cache.B, desc.Hq)
    assert q.is_contiguous() and out.is_contiguous() and q.dtype is cache.dtype and out.dtype is torch.float32
    assert q.shape == out.shape == (*heads, desc.D) and desc.B == cache.B
    *lists, entries = idx.shape
    assert idx.dtype is count.dtype is torch.int32 and tuple(lists) == count.shape == heads and count.is_contiguous()
    idx_b, idx_h, idx_n = idx.stride()
    assert max_count <= entries and (entries < 2 or idx_n == 1) and (heads[0] < 2 or idx_b == heads[1] * idx_h)
    assert lse is None or (lse.dtype is torch.float32 and lse.shape == heads and lse.is_contiguous())
    rc = (_lib or load_library()).tb_sparse_decode_attn_paged(
        ctypes.byref(desc), cache.ref, q.data_ptr(), idx.data_ptr(), count.data_ptr(), idx_h, max_count, tail_begin, tail_end, sm_scale,
        out.data_ptr(), None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.nbytes,
        _stream_on(cache.device, stream, (q, idx, count, out, lse, ws) if _several_devices else ()))
    if rc:
        _check(rc, "tb_sparse_decode_attn_paged")


def policy_count(N: int, k: int, sink: int, window: int) -> int:
    """Length of the list the selection policy emits (host-side sizing helper)."""
    lo = min(sink, N)
    hi = max(lo, N - window)
    return lo + min(k, hi - lo) + (N - hi)
