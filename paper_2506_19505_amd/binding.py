"""ctypes binding with the same names as the C ABI (include/antkv.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libantkv.so")
_lib = None

EXPORTS = (
    "antkv_version", "antkv_strerror", "antkv_encode", "antkv_anchor_select_workspace", "antkv_anchor_select",
    "antkv_topk_workspace", "antkv_topk", "antkv_gather_rows", "antkv_decode_attn_workspace", "antkv_decode_attn",
    "antkv_decode_attn_static", "antkv_set_decode_options", "antkv_decode_attn_prerope_workspace", "antkv_decode_attn_prerope", "antkv_append_token", "antkv_prefill_attn", "antkv_kmeans_step_workspace", "antkv_kmeans_step",
    "antkv_prefill_attn_window", "antkv_page_map", "antkv_page_store", "antkv_page_load", "antkv_page_attn_workspace", "antkv_page_attn",
    "antkv_qpage_store", "antkv_qpage_load", "antkv_qpage_attn_workspace", "antkv_qpage_attn", "antkv_rope_freqs", "antkv_rope",
)


class AntkvError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: error {code} ({_strerror(code)})")
        self.code = code


class _Geom(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "D", "d_sub", "n_centroids")]


@dataclass(frozen=True)
class Geometry:
    B: int
    Hq: int
    Hkv: int
    d_sub: int
    D: int = 128
    n_centroids: int = 256

    @property
    def M(self) -> int:
        return self.D // self.d_sub

    @property
    def code_bytes(self) -> int:
        """Bytes of one token's codes: one byte per sub-space, or the M 12-bit codes packed (4096 centroids)."""
        return self.M if self.n_centroids <= 256 else (self.M * 12 + 7) // 8

    def c(self) -> _Geom:
        return _Geom(self.B, self.Hq, self.Hkv, self.D, self.d_sub, self.n_centroids)

    @functools.cached_property
    def _c(self) -> _Geom:
        """Built on first use: a call passes it by reference and only reads it."""
        return self.c()


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libantkv.so; fails loudly if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2506_19505_amd.build` "
                              "(or __graft_entry__.build()); the AnTKV path has no CPU fallback")
        lib = ctypes.CDLL(_LIB_PATH)
        i64, vp, sz, f32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
        gp = ctypes.POINTER(_Geom)
        lib.antkv_version.restype = ctypes.c_int
        lib.antkv_strerror.restype = ctypes.c_char_p
        lib.antkv_strerror.argtypes = [ctypes.c_int]
        lib.antkv_encode.restype = ctypes.c_int
        lib.antkv_encode.argtypes = [gp, vp, i64, i64, i64, i64, vp, vp, i64, i64, vp]
        lib.antkv_anchor_select_workspace.restype = sz
        lib.antkv_anchor_select_workspace.argtypes = [gp, i64, i64, i64]
        lib.antkv_anchor_select.restype = ctypes.c_int
        lib.antkv_anchor_select.argtypes = [gp, vp, vp, i64, i64, f32, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.antkv_topk_workspace.restype = sz
        lib.antkv_topk_workspace.argtypes = [i64, i64, i64]
        lib.antkv_topk.restype = ctypes.c_int
        lib.antkv_topk.argtypes = [vp, i64, i64, i64, vp, vp, sz, vp]
        lib.antkv_gather_rows.restype = ctypes.c_int
        lib.antkv_gather_rows.argtypes = [gp, vp, i64, vp, i64, vp, vp]
        lib.antkv_kmeans_step_workspace.restype = sz
        lib.antkv_kmeans_step_workspace.argtypes = [gp]
        lib.antkv_kmeans_step.restype = ctypes.c_int
        lib.antkv_kmeans_step.argtypes = [gp, vp, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.antkv_prefill_attn.restype = ctypes.c_int
        lib.antkv_prefill_attn.argtypes = [gp, vp, vp, vp, i64, i64, f32, vp, vp, vp, vp]
        lib.antkv_append_token.restype = ctypes.c_int
        lib.antkv_append_token.argtypes = [gp, vp, vp, i64, i64, vp, vp, vp, vp, i64, vp, vp, i64, vp, vp, i64, vp]
        lib.antkv_decode_attn_workspace.restype = sz
        lib.antkv_decode_attn_workspace.argtypes = [gp, i64, i64, i64, i64]
        lib.antkv_decode_attn.restype = ctypes.c_int
        lib.antkv_decode_attn.argtypes = [gp, vp, f32, vp, vp, i64, i64, vp, vp, vp, vp, i64, vp, vp, i64, vp,
                                          vp, vp, vp, vp, i64, vp, sz, vp]
        lib.antkv_decode_attn_static.restype = ctypes.c_int
        lib.antkv_decode_attn_static.argtypes = [gp, vp, f32, vp, vp, i64, i64, vp, vp, vp, vp, i64, vp, vp, i64, vp, vp]
        lib.antkv_set_decode_options.restype = ctypes.c_int
        lib.antkv_set_decode_options.argtypes = [ctypes.c_int]
        lib.antkv_decode_attn_prerope_workspace.restype = sz
        lib.antkv_decode_attn_prerope_workspace.argtypes = [gp, i64, i64]
        lib.antkv_decode_attn_prerope.restype = ctypes.c_int
        lib.antkv_decode_attn_prerope.argtypes = [gp, vp, f32, vp, vp, i64, i64, vp, vp, vp, vp, i64, vp, vp, i64,
                                                  f32, ctypes.c_int, i64, vp, vp, sz, vp]
        i32 = ctypes.c_int32
        lib.antkv_prefill_attn_window.restype = ctypes.c_int
        lib.antkv_prefill_attn_window.argtypes = [gp, vp, vp, vp, i64, i64, f32, i64, i64, vp, vp, vp, vp]
        lib.antkv_page_map.restype = ctypes.c_int
        lib.antkv_page_map.argtypes = [i64, vp, vp, vp, i64, i64, i32, vp, i64, vp, i64, vp, vp, vp, vp, vp]
        lib.antkv_page_store.restype = ctypes.c_int
        lib.antkv_page_store.argtypes = [gp, vp, vp, i64, i64, i64, vp, vp, vp, i64, i32, vp]
        lib.antkv_page_load.restype = ctypes.c_int
        lib.antkv_page_load.argtypes = [gp, vp, vp, i64, i32, vp, i64, vp, i64, i64, vp, vp, i64, i64, i64, vp]
        lib.antkv_page_attn_workspace.restype = sz
        lib.antkv_page_attn_workspace.argtypes = [gp, i64]
        lib.antkv_page_attn.restype = ctypes.c_int
        lib.antkv_page_attn.argtypes = [gp, vp, i64, i64, i64, vp, vp, vp, i64, vp, vp, i64, i32, f32, i64, i64, vp, vp, vp, vp, sz, vp]
        lib.antkv_qpage_store.restype = ctypes.c_int
        lib.antkv_qpage_store.argtypes = [gp, vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, i64, i32, vp]
        lib.antkv_qpage_load.restype = ctypes.c_int
        lib.antkv_qpage_load.argtypes = [gp, vp, vp, vp, vp, i64, i32, vp, i64, vp, i64, i64, vp, vp, i64, i64, i64, i32, vp]
        lib.antkv_qpage_attn_workspace.restype = sz
        lib.antkv_qpage_attn_workspace.argtypes = [gp, i64]
        lib.antkv_qpage_attn.restype = ctypes.c_int
        lib.antkv_qpage_attn.argtypes = [gp, vp, i64, i64, i64, vp, vp, vp, i64, vp, vp, vp, vp, i64, i32, f32, i64, i64, vp, vp, vp, vp, sz, vp]
        f64 = ctypes.c_double
        lib.antkv_rope_freqs.restype = ctypes.c_int
        lib.antkv_rope_freqs.argtypes = [i32, f64, f64, f64, f64, f64, vp, vp]
        lib.antkv_rope.restype = ctypes.c_int
        lib.antkv_rope.argtypes = [gp, vp, i64, i64, i64, vp, i64, i64, i64, i64, vp, vp, vp, i64, vp, i32, i32, f32, i32, vp, i64, i64, i64, vp, i64, i64, i64, vp]
        _lib = lib
    return _lib


def _strerror(code: int) -> str:
    return load_library().antkv_strerror(code).decode()


def version() -> int:
    return int(load_library().antkv_version())


# Host cost of a call: argument conversion, the stream and the checks took 6 us of the 9.5 us of a decode_attn call when
# every argument became a c_void_p and the stream came through torch.cuda.current_stream (2 us by itself).  Addresses go as
# plain ints (ctypes converts them by argtypes) and the stream's handle is asked for directly: 5 us, launch included.
def _p(t):
    return None if t is None else t.data_ptr()


def _stream(t: torch.Tensor):
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _check(rc: int, what: str):
    if rc != 0:
        raise AntkvError(rc, what)


def _need(t: torch.Tensor, dtype, name: str):
    if t.is_cuda and t.dtype is dtype and t.is_contiguous():
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def encode(geom: Geometry, x: torch.Tensor, codebook: torch.Tensor, codes: torch.Tensor | None = None,
           token_offset: int = 0) -> torch.Tensor:
    """antkv_encode: x fp16 [B,Hkv,n,D] (last dim contiguous) -> codes uint8 [B,Hkv,N_cap,M]."""
    if not x.is_cuda or x.dtype != torch.float16 or x.stride(-1) != 1:
        raise ValueError("x must be an fp16 device tensor with contiguous channels")
    _need(codebook, torch.float16, "codebook")
    B, Hkv, n, _ = x.shape
    if codes is None:
        codes = torch.empty((B, Hkv, n, geom.code_bytes), dtype=torch.uint8, device=x.device)
    _need(codes, torch.uint8, "codes")
    rc = load_library().antkv_encode(geom._c, _p(x), x.stride(0), x.stride(1), x.stride(2), n, _p(codebook),
                                     _p(codes), codes.shape[2], token_offset, _stream(x))
    _check(rc, "antkv_encode")
    return codes


def topk(scores: torch.Tensor, k: int) -> torch.Tensor:
    """antkv_topk: scores fp32 [..., N] -> idx int32 [..., k]."""
    _need(scores, torch.float32, "scores")
    N = scores.shape[-1]
    rows = scores.numel() // max(N, 1)
    idx = torch.empty(scores.shape[:-1] + (k,), dtype=torch.int32, device=scores.device)
    lib = load_library()
    ws = _workspace(lib.antkv_topk_workspace(rows, N, k), scores.device)
    rc = lib.antkv_topk(_p(scores), rows, N, k, _p(idx), _p(ws), ws.numel(), _stream(scores))
    _check(rc, "antkv_topk")
    return idx


def kmeans_step(geom: Geometry, x: torch.Tensor, w: torch.Tensor, codebook: torch.Tensor):
    """antkv_kmeans_step: x fp16 [B,Hkv,n,D], w fp32 [B,Hkv,n], codebook fp16 [Hkv,M,C,d] ->
    (new codebook fp16, codes uint8 [B,Hkv,n,code_bytes], wsum fp32 [Hkv,M,C], objective fp64 [Hkv,M])."""
    _need(x, torch.float16, "x")
    _need(w, torch.float32, "w")
    _need(codebook, torch.float16, "codebook")
    B, Hkv, n, _ = x.shape
    dev = x.device
    out = torch.empty_like(codebook)
    codes = torch.empty((B, Hkv, n, geom.code_bytes), dtype=torch.uint8, device=dev)
    wsum = torch.empty((Hkv, geom.M, geom.n_centroids), dtype=torch.float32, device=dev)
    objective = torch.empty((Hkv, geom.M), dtype=torch.float64, device=dev)
    lib = load_library()
    ws = _workspace(lib.antkv_kmeans_step_workspace(geom._c), dev)
    rc = lib.antkv_kmeans_step(geom._c, _p(x), _p(w), n, _p(codebook), _p(out), _p(codes), _p(wsum),
                               _p(objective), _p(ws), ws.numel(), _stream(x))
    _check(rc, "antkv_kmeans_step")
    return out, codes, wsum, objective


def prefill_attn(geom: Geometry, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float,
                 want_stats: bool = True):
    """antkv_prefill_attn: q fp16 [B,Hq,Nq,D], k / v fp16 [B,Hkv,N,D] -> (out fp16 [B,Hq,Nq,D], row_max, row_sum)."""
    _need(q, torch.float16, "q")
    _need(k, torch.float16, "k")
    _need(v, torch.float16, "v")
    B, Hq, Nq, D = q.shape
    N = k.shape[2]
    out = torch.empty((B, Hq, Nq, D), dtype=torch.float16, device=q.device)
    row_max = torch.empty((B, Hq, Nq), dtype=torch.float32, device=q.device) if want_stats else None
    row_sum = torch.empty((B, Hq, Nq), dtype=torch.float32, device=q.device) if want_stats else None
    rc = load_library().antkv_prefill_attn(geom._c, _p(q), _p(k), _p(v), N, Nq, float(scale), _p(out),
                                           _p(row_max), _p(row_sum), _stream(q))
    _check(rc, "antkv_prefill_attn")
    return out, row_max, row_sum


def anchor_select(geom: Geometry, q: torch.Tensor, k_fp16: torch.Tensor, scale: float, k: int,
                  row_max: torch.Tensor | None = None, row_sum: torch.Tensor | None = None,
                  want_scores: bool = True):
    """antkv_anchor_select: q fp16 [B,Hq,Nq,D], k fp16 [B,Hkv,N,D] -> (idx_k, idx_v, ans_k, ans_v)."""
    _need(q, torch.float16, "q")
    _need(k_fp16, torch.float16, "k_fp16")
    B, Hkv, N, _ = k_fp16.shape
    Nq = q.shape[2]
    dev = q.device
    ans_k = torch.empty((B, Hkv, N), dtype=torch.float32, device=dev) if want_scores else None
    ans_v = torch.empty((B, Hkv, N), dtype=torch.float32, device=dev) if want_scores else None
    idx_k = torch.empty((B, Hkv, k), dtype=torch.int32, device=dev)
    idx_v = torch.empty((B, Hkv, k), dtype=torch.int32, device=dev)
    lib = load_library()
    ws = _workspace(lib.antkv_anchor_select_workspace(geom._c, N, Nq, k), dev)
    rc = lib.antkv_anchor_select(geom._c, _p(q), _p(k_fp16), N, Nq, float(scale), k, _p(row_max), _p(row_sum),
                                 _p(ans_k), _p(ans_v), _p(idx_k), _p(idx_v), _p(ws), ws.numel(), _stream(q))
    _check(rc, "antkv_anchor_select")
    return idx_k, idx_v, ans_k, ans_v


def gather_rows(geom: Geometry, x: torch.Tensor, idx: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """antkv_gather_rows: x fp16 [B,Hkv,N,D], idx int32 [B,Hkv,k] -> rows fp16 [B,Hkv,k,D]."""
    _need(x, torch.float16, "x")
    _need(idx, torch.int32, "idx")
    B, Hkv, N, D = x.shape
    k = idx.shape[-1]
    if out is None:
        out = torch.empty((B, Hkv, k, D), dtype=torch.float16, device=x.device)
    _need(out, torch.float16, "out")
    rows = out
    rc = load_library().antkv_gather_rows(geom._c, _p(x), N, _p(idx), k, _p(rows), _stream(x))
    _check(rc, "antkv_gather_rows")
    return rows


def append_token(geom: Geometry, k_new: torch.Tensor, v_new: torch.Tensor, N: int, W: int, cb_k: torch.Tensor,
                 cb_v: torch.Tensor, codes_k: torch.Tensor, codes_v: torch.Tensor, idx_k: torch.Tensor | None,
                 rows_k: torch.Tensor | None, idx_v: torch.Tensor | None, rows_v: torch.Tensor | None) -> int:
    """antkv_append_token: retire the oldest of the W window tokens into the codes, shift the window (the last W
    entries of both anchor lists) and append the new rows at position N.  Returns the new context length N + 1."""
    _need(k_new, torch.float16, "k_new")
    _need(v_new, torch.float16, "v_new")
    _need(codes_k, torch.uint8, "codes_k")
    _need(codes_v, torch.uint8, "codes_v")
    k_k = 0 if idx_k is None else idx_k.shape[-1]
    k_v = 0 if idx_v is None else idx_v.shape[-1]
    for name, t, dt in (("idx_k", idx_k, torch.int32), ("rows_k", rows_k, torch.float16), ("idx_v", idx_v, torch.int32),
                        ("rows_v", rows_v, torch.float16)):
        if t is not None:
            _need(t, dt, name)
    rc = load_library().antkv_append_token(
        geom._c, _p(k_new), _p(v_new), N, W, _p(cb_k), _p(cb_v), _p(codes_k), _p(codes_v), codes_k.shape[2],
        _p(idx_k), _p(rows_k), k_k, _p(idx_v), _p(rows_v), k_v, _stream(k_new))
    _check(rc, "antkv_append_token")
    return N + 1


class DecodeWorkspace:
    """Caller-owned scratch for antkv_decode_attn, sized once and reused across calls."""

    def __init__(self, geom: Geometry, N: int, k_k: int, k_v: int, k_resel: int, device):
        self.nbytes = load_library().antkv_decode_attn_workspace(geom._c, N, k_k, k_v, k_resel)
        self.buf = _workspace(self.nbytes, device)


def decode_attn(geom: Geometry, q: torch.Tensor, scale: float, codes_k: torch.Tensor, codes_v: torch.Tensor,
                cb_k: torch.Tensor, cb_v: torch.Tensor, idx_k: torch.Tensor | None, rows_k: torch.Tensor | None,
                idx_v: torch.Tensor | None, rows_v: torch.Tensor | None, N: int | None = None,
                out: torch.Tensor | None = None, want_ans: bool = False, k_resel: int = 0,
                workspace: DecodeWorkspace | None = None):
    """antkv_decode_attn.  Returns out fp16 [B,Hq,D], or (out, ans_k, ans_v, resel_idx_k, resel_idx_v)."""
    _need(q, torch.float16, "q")
    _need(codes_k, torch.uint8, "codes_k")
    _need(codes_v, torch.uint8, "codes_v")
    dev = q.device
    B, Hq, D = q.shape
    Hkv = geom.Hkv
    N_cap = codes_k.shape[2]
    if N is None:
        N = N_cap
    k_k = 0 if idx_k is None else idx_k.shape[-1]
    k_v = 0 if idx_v is None else idx_v.shape[-1]
    if out is None:
        out = torch.empty((B, Hq, D), dtype=torch.float16, device=dev)
    ans_k = ans_v = rk = rv = None
    if want_ans or k_resel > 0:
        ans_k = torch.empty((B, Hkv, N), dtype=torch.float32, device=dev)
        ans_v = torch.empty((B, Hkv, N), dtype=torch.float32, device=dev)
    if k_resel > 0:
        rk = torch.empty((B, Hkv, k_resel), dtype=torch.int32, device=dev)
        rv = torch.empty((B, Hkv, k_resel), dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = DecodeWorkspace(geom, N, k_k, k_v, k_resel, dev)
    rc = load_library().antkv_decode_attn(
        geom._c, _p(q), float(scale), _p(codes_k), _p(codes_v), N, N_cap, _p(cb_k), _p(cb_v),
        _p(idx_k) if k_k else None, _p(rows_k) if k_k else None, k_k,
        _p(idx_v) if k_v else None, _p(rows_v) if k_v else None, k_v,
        _p(out), _p(ans_k), _p(ans_v), _p(rk), _p(rv), k_resel, _p(workspace.buf), workspace.buf.numel(), _stream(q))
    _check(rc, "antkv_decode_attn")
    if want_ans or k_resel > 0:
        return out, ans_k, ans_v, rk, rv
    return out


def decode_attn_prerope_workspace(geom: Geometry, N: int, k_v: int, device) -> torch.Tensor:
    """A workspace of antkv_decode_attn_prerope_workspace(geom, N, k_v) bytes for decode_attn_prerope."""
    return _workspace(load_library().antkv_decode_attn_prerope_workspace(geom._c, N, k_v), device)


def decode_attn_prerope(geom: Geometry, q: torch.Tensor, scale: float, codes_k: torch.Tensor, codes_v: torch.Tensor,
                        cb_k: torch.Tensor, cb_v: torch.Tensor, idx_k: torch.Tensor | None, rows_k: torch.Tensor | None,
                        idx_v: torch.Tensor | None, rows_v: torch.Tensor | None, rope_base: float = 10000.0,
                        rope_style: int = 0, pos0: int = 0, N: int | None = None, out: torch.Tensor | None = None,
                        workspace: torch.Tensor | None = None) -> torch.Tensor:
    """antkv_decode_attn_prerope: decode attention on keys stored before RoPE.  Returns out fp16 [B,Hq,D]."""
    _need(q, torch.float16, "q")
    _need(codes_k, torch.uint8, "codes_k")
    _need(codes_v, torch.uint8, "codes_v")
    B, Hq, D = q.shape
    N_cap = codes_k.shape[2]
    if N is None:
        N = N_cap
    k_k = 0 if idx_k is None else idx_k.shape[-1]
    k_v = 0 if idx_v is None else idx_v.shape[-1]
    if out is None:
        out = torch.empty((B, Hq, D), dtype=torch.float16, device=q.device)
    if workspace is None:
        workspace = decode_attn_prerope_workspace(geom, N, k_v, q.device)
    rc = load_library().antkv_decode_attn_prerope(
        geom._c, _p(q), float(scale), _p(codes_k), _p(codes_v), N, N_cap, _p(cb_k), _p(cb_v),
        _p(idx_k) if k_k else None, _p(rows_k) if k_k else None, k_k,
        _p(idx_v) if k_v else None, _p(rows_v) if k_v else None, k_v,
        float(rope_base), int(rope_style), int(pos0), _p(out), _p(workspace), workspace.numel(), _stream(q))
    _check(rc, "antkv_decode_attn_prerope")
    return out


DECODE_FIXED_ORDER, DECODE_WIDE_TABLE = 1, 2     # ANTKV_DECODE_* of include/antkv.h


def set_decode_options(options: int) -> int:
    """antkv_set_decode_options: process-wide option mask of the one-byte-code decode kernel (DECODE_FIXED_ORDER for a
    bit-reproducible output, DECODE_WIDE_TABLE for 30-bit table entries).  Returns the previous mask."""
    return int(load_library().antkv_set_decode_options(int(options)))


STATIC_SCRATCH_BYTES = 8 << 20     # ANTKV_STATIC_SCRATCH_BYTES of include/antkv.h


def decode_attn_static(geom: Geometry, q: torch.Tensor, scale: float, codes_k: torch.Tensor, codes_v: torch.Tensor,
                       cb_k: torch.Tensor, cb_v: torch.Tensor, idx_k: torch.Tensor | None, rows_k: torch.Tensor | None,
                       idx_v: torch.Tensor | None, rows_v: torch.Tensor | None, out: torch.Tensor,
                       N: int | None = None) -> torch.Tensor:
    """antkv_decode_attn_static: decode attention with the scratch inside the library.  `out` is the caller's
    fp16 [B,Hq,D] tensor (this wrapper allocates nothing either)."""
    _need(q, torch.float16, "q")
    _need(codes_k, torch.uint8, "codes_k")
    _need(codes_v, torch.uint8, "codes_v")
    _need(out, torch.float16, "out")
    N_cap = codes_k.shape[2]
    if N is None:
        N = N_cap
    k_k = 0 if idx_k is None else idx_k.shape[-1]
    k_v = 0 if idx_v is None else idx_v.shape[-1]
    rc = load_library().antkv_decode_attn_static(
        geom._c, _p(q), float(scale), _p(codes_k), _p(codes_v), N, N_cap, _p(cb_k), _p(cb_v),
        _p(idx_k) if k_k else None, _p(rows_k) if k_k else None, k_k,
        _p(idx_v) if k_v else None, _p(rows_v) if k_v else None, k_v, _p(out), _stream(q))
    _check(rc, "antkv_decode_attn_static")
    return out


# ---- the FP16 cache in pages, and windowed prompts ----------------------------------------------------------------------
# Host cost of a call: checks by keyword arguments and generators took 4 of the 9.8 us of a page_store call and, with four outputs
# allocated one by one, 9 of the 15 us of page_map.  Each check now asks first whether all is well.

def _run(call, what: str, device: int, *args):
    """The call on `device`, which is made current for it if it is not."""
    if torch._C._cuda_getDevice() == device:
        rc = call(*args)
    else:
        with torch.cuda.device(device):
            rc = call(*args)
    if rc != 0:
        raise AntkvError(rc, what)


def _one_device(*tensors) -> int:
    at = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ValueError("all tensors must be on the same device")
    return at


def _rows(t: torch.Tensor, name: str, heads: int):
    """fp16 [T, heads, D] with contiguous channels; any strides of tokens and heads."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype is not torch.float16:
        raise TypeError(f"{name} must be torch.float16")
    if t.dim() != 3 or t.shape[1:] != (heads, 128) or t.stride(2) != 1:
        raise ValueError(f"{name} must be [T, {heads}, 128] with contiguous channels")


def _pools(k_pages: torch.Tensor, v_pages: torch.Tensor, heads: int):
    _need(k_pages, torch.float16, "k_pages")
    _need(v_pages, torch.float16, "v_pages")
    shape = k_pages.shape
    if len(shape) != 4 or shape[1] != heads or shape[3] != 128 or v_pages.shape != shape:
        raise ValueError(f"k_pages and v_pages must be [n_pages, {heads}, page_size, 128]")
    return shape[0], shape[2]


def _ints(t: torch.Tensor, name: str, shape: tuple):
    _need(t, torch.int32, name)
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {list(shape)}")


def _table(t: torch.Tensor, requests: int) -> int:
    _need(t, torch.int32, "table")
    if t.dim() != 2 or t.shape[0] != requests:
        raise ValueError(f"table must be [{requests}, entries]")
    return t.shape[1]


def prefill_attn_window(geom: Geometry, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float, window: int, n_sink: int = 0,
                        want_stats: bool = True):
    """antkv_prefill_attn_window: prefill_attn in which a query sees the last `window` positions and the first `n_sink`.
    q fp16 [B,Hq,Nq,D], k / v fp16 [B,Hkv,N,D] -> (out fp16 [B,Hq,Nq,D], row_max, row_sum).  The statistics are of the keys that a row
    sees: not for anchor_select where the window hides some."""
    _need(q, torch.float16, "q")
    _need(k, torch.float16, "k")
    _need(v, torch.float16, "v")
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k and v must have four dimensions")
    B, Hq, Nq, D = q.shape
    N = k.shape[2]
    if (B, Hq, D) != (geom.B, geom.Hq, geom.D) or k.shape != (B, geom.Hkv, N, D) or v.shape != k.shape:
        raise ValueError("q, k and v do not fit the geometry")
    device = _one_device(q, k, v)
    out = torch.empty_like(q)
    row_max = row_sum = None
    if want_stats:
        row_max, row_sum = torch.empty((2, B, Hq, Nq), dtype=torch.float32, device=q.device).unbind(0)
    _run(load_library().antkv_prefill_attn_window, "antkv_prefill_attn_window", device, geom._c, q.data_ptr(), k.data_ptr(), v.data_ptr(), N, Nq,
         float(scale), int(window), int(n_sink), out.data_ptr(), _p(row_max), _p(row_sum), _stream(q))
    return out, row_max, row_sum


def page_map(held_len: torch.Tensor, new_len: torch.Tensor, table: torch.Tensor, page_size: int, n_pages: int, free_pages: torch.Tensor,
             T: int, free_at: torch.Tensor | None = None, out=None):
    """antkv_page_map: held_len, new_len int32 [R], table int32 [R,cap] (new entries are written), free_pages int32 [n] ->
    (ctx_len int32 [R], q_start int32 [R+1], slot int32 [T], status int32 [2]).  `out`: such a tuple, to be written again."""
    R = held_len.shape[0]
    _ints(held_len, "held_len", (R,))
    _ints(new_len, "new_len", (R,))
    cap = _table(table, R)
    _need(free_pages, torch.int32, "free_pages")
    if free_at is not None:
        _need(free_at, torch.int32, "free_at")
        if free_at.numel() < 1:
            raise ValueError("free_at must hold a number")
    if out is None:
        slot, ctx_len, q_start, status = table.new_empty(T + 2 * R + 3).split_with_sizes((T, R, R + 1, 2))
        out = ctx_len, q_start, slot, status
        device = _one_device(table, held_len, new_len, free_pages, free_at)
    else:
        ctx_len, q_start, slot, status = out
        _ints(ctx_len, "ctx_len", (R,))
        _ints(q_start, "q_start", (R + 1,))
        _ints(slot, "slot", (T,))
        _ints(status, "status", (2,))
        device = _one_device(table, held_len, new_len, free_pages, free_at, *out)
    _run(load_library().antkv_page_map, "antkv_page_map", device, R, held_len.data_ptr(), new_len.data_ptr(), table.data_ptr(), cap, n_pages, page_size,
         free_pages.data_ptr(), free_pages.numel(), _p(free_at), T, ctx_len.data_ptr(), q_start.data_ptr(), slot.data_ptr(), status.data_ptr(),
         _stream(table))
    return out


def page_store(geom: Geometry, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor) -> None:
    """antkv_page_store: rows of k, v fp16 [T,Hkv,D] (equal strides, channels contiguous) to slot int32 [T] of the pools
    fp16 [n_pages,Hkv,page_size,D]."""
    heads = geom.Hkv
    _rows(k, "k", heads)
    n_pages, page_size = _pools(k_pages, v_pages, heads)
    T = k.shape[0]
    if v.shape != k.shape or v.stride() != k.stride() or v.dtype is not torch.float16:
        _rows(v, "v", heads)
        if v.shape[0] != T or (T > 1 and v.stride(0) != k.stride(0)) or (heads > 1 and v.stride(1) != k.stride(1)):
            raise ValueError("k and v must have the same shape and strides")
    _ints(slot, "slot", (T,))
    _run(load_library().antkv_page_store, "antkv_page_store", _one_device(k_pages, v_pages, k, v, slot), geom._c, k.data_ptr(), v.data_ptr(),
         k.stride(0) if T > 1 else 0, k.stride(1) if heads > 1 else 0, T, slot.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), n_pages, page_size,
         _stream(k_pages))


def page_load(geom: Geometry, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, N: int, first: int = 0,
              ctx_len: torch.Tensor | None = None, k: torch.Tensor | None = None, v: torch.Tensor | None = None):
    """antkv_page_load: positions first .. first + N - 1 of the table's requests -> (k, v) fp16 [B,Hkv,N,D].  Rows at or behind
    ctx_len (int32 [B]) are left as they are: zeros where k and v are made here."""
    n_pages, page_size = _pools(k_pages, v_pages, geom.Hkv)
    cap = _table(table, geom.B)
    if ctx_len is not None:
        _ints(ctx_len, "ctx_len", (geom.B,))
    shape = (geom.B, geom.Hkv, N, geom.D)
    if k is None:
        k = torch.zeros(shape, dtype=torch.float16, device=k_pages.device)
    if v is None:
        v = torch.zeros(shape, dtype=torch.float16, device=k_pages.device)
    _need(k, torch.float16, "k")
    _need(v, torch.float16, "v")
    if k.shape != shape or v.shape != shape:
        raise ValueError(f"k and v must be {list(shape)}")
    rows = N * geom.D
    _run(load_library().antkv_page_load, "antkv_page_load", _one_device(k_pages, v_pages, table, ctx_len, k, v), geom._c, k_pages.data_ptr(),
         v_pages.data_ptr(), n_pages, page_size, table.data_ptr(), cap, _p(ctx_len), first, N, k.data_ptr(), v.data_ptr(), geom.Hkv * rows, rows,
         geom.D, _stream(k_pages))
    return k, v


def page_attn_workspace(geom: Geometry, T: int, device) -> torch.Tensor:
    """A workspace of antkv_page_attn_workspace(geom, T) bytes for page_attn, for calls that follow each other on one stream with up to
    T rows."""
    nbytes = load_library().antkv_page_attn_workspace(geom._c, T)
    if nbytes == 0 and T != 0 and geom.B != 0:
        raise ValueError(f"page_attn does not take {T} rows of this geometry")
    return _workspace(nbytes, device)


def page_attn(geom: Geometry, q: torch.Tensor, scale: float, q_start: torch.Tensor, ctx_len: torch.Tensor, table: torch.Tensor,
              k_pages: torch.Tensor, v_pages: torch.Tensor, window: int = 0, n_sink: int = 0, out: torch.Tensor | None = None,
              want_stats: bool = False, workspace: torch.Tensor | None = None):
    """antkv_page_attn: q fp16 [T,Hq,D] (channels contiguous), q_start int32 [R+1], ctx_len int32 [R], table int32 [R,cap], pools
    fp16 [n_pages,Hkv,page_size,D], geom.B = R -> (out fp16 [T,Hq,D], row_max, row_sum fp32 [Hq,T] or None).
    Rows of out behind q_start[R] are left as they are (undefined where out is made here).  The statistics are of the keys that a row sees:
    not for anchor_select where a window hides some."""
    Hq, R = geom.Hq, geom.B
    _rows(q, "q", Hq)
    n_pages, page_size = _pools(k_pages, v_pages, geom.Hkv)
    T = q.shape[0]
    _ints(q_start, "q_start", (R + 1,))
    _ints(ctx_len, "ctx_len", (R,))
    cap = _table(table, R)
    if out is None:
        out = k_pages.new_empty((T, Hq, 128))
    else:
        _need(out, torch.float16, "out")
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    row_max = row_sum = None
    if want_stats:
        row_max, row_sum = torch.empty((2, Hq, T), dtype=torch.float32, device=q.device).unbind(0)
    if workspace is None:
        workspace = _workspace(load_library().antkv_page_attn_workspace(geom._c, T), q.device)
    else:
        _need(workspace, torch.uint8, "workspace")
    _run(load_library().antkv_page_attn, "antkv_page_attn", _one_device(q, k_pages, v_pages, q_start, ctx_len, table, out, workspace), geom._c,
         q.data_ptr(), q.stride(0) if T > 1 else 0, q.stride(1) if Hq > 1 else 0, T, q_start.data_ptr(), ctx_len.data_ptr(), table.data_ptr(), cap,
         k_pages.data_ptr(), v_pages.data_ptr(), n_pages, page_size, float(scale), int(window), int(n_sink), out.data_ptr(), _p(row_max), _p(row_sum),
         workspace.data_ptr(), workspace.numel(), _stream(q))
    return out, row_max, row_sum


# ---- the same cache in 8 bits -------------------------------------------------------------------------------------------

# Host cost of a call: with every check a function call of its own, 4.5 of the 11.3 us of qpage_attn.  Below each call asks in one go whether
# all is well, and only otherwise what is wrong.

_E4M3, _HALF, _FLOAT, _INT = torch.float8_e4m3fn, torch.float16, torch.float32, torch.int32


def _byte_pools(k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor, heads: int):
    """-> n_pages, page_size, device"""
    shape, device = k_pages.shape, k_pages.get_device()
    if (k_pages.dtype is _E4M3 and v_pages.dtype is _E4M3 and k_scales.dtype is _FLOAT and v_scales.dtype is _FLOAT and len(shape) == 4
            and v_pages.shape == shape and device >= 0 and device == v_pages.get_device() == k_scales.get_device() == v_scales.get_device()):
        n_pages, h, page_size, d = shape
        if (h == heads and d == 128 and k_scales.shape == (n_pages, heads, page_size // 16) and v_scales.shape == k_scales.shape
                and k_pages.is_contiguous() and v_pages.is_contiguous() and k_scales.is_contiguous() and v_scales.is_contiguous()):
            return n_pages, page_size, device
    _need(k_pages, _E4M3, "k_pages")
    _need(v_pages, _E4M3, "v_pages")
    _need(k_scales, _FLOAT, "k_scales")
    _need(v_scales, _FLOAT, "v_scales")
    if len(shape) != 4 or shape[1] != heads or shape[3] != 128 or v_pages.shape != shape:
        raise ValueError(f"k_pages and v_pages must be [n_pages, {heads}, page_size, 128]")
    if k_scales.shape != (shape[0], heads, shape[2] // 16) or v_scales.shape != k_scales.shape:
        raise ValueError(f"k_scales and v_scales must be [{shape[0]}, {heads}, {shape[2] // 16}]")
    raise ValueError("all tensors must be on the same device")


def _on(device: int, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("all tensors must be on the same device" if t.is_cuda else "all tensors must be device tensors")


def qpage_store(geom: Geometry, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor,
                v_scales: torch.Tensor) -> None:
    """antkv_qpage_store: rows of k, v fp16 [T,Hkv,D] (equal strides, channels contiguous) to slot int32 [T] of pools
    float8_e4m3fn [n_pages,Hkv,page_size,D] with scales fp32 [n_pages,Hkv,page_size/16]."""
    heads = geom.Hkv
    _rows(k, "k", heads)
    n_pages, page_size, device = _byte_pools(k_pages, v_pages, k_scales, v_scales, heads)
    T, strides = k.shape[0], k.stride()
    if v.shape != k.shape or v.stride() != strides or v.dtype is not _HALF:
        _rows(v, "v", heads)
        if v.shape[0] != T or (T > 1 and v.stride(0) != strides[0]) or (heads > 1 and v.stride(1) != strides[1]):
            raise ValueError("k and v must have the same shape and strides")
    if slot.dtype is not _INT or slot.shape != (T,) or not slot.is_contiguous():
        _ints(slot, "slot", (T,))
    _on(device, k, v, slot)
    _run(load_library().antkv_qpage_store, "antkv_qpage_store", device, geom._c, k.data_ptr(),
         v.data_ptr(), strides[0] if T > 1 else 0, strides[1] if heads > 1 else 0, T, slot.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
         k_scales.data_ptr(), v_scales.data_ptr(), n_pages, page_size, _stream(k_pages))


def qpage_load(geom: Geometry, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor, table: torch.Tensor, N: int,
               first: int = 0, ctx_len: torch.Tensor | None = None, k: torch.Tensor | None = None, v: torch.Tensor | None = None):
    """antkv_qpage_load: positions first .. first + N - 1 of the table's requests -> (k, v) fp16 [B,Hkv,N,D].  Rows at or behind
    ctx_len (int32 [B]) are left as they are: zeros where k and v are made here."""
    n_pages, page_size, device = _byte_pools(k_pages, v_pages, k_scales, v_scales, geom.Hkv)
    cap = _table(table, geom.B)
    if ctx_len is not None:
        _ints(ctx_len, "ctx_len", (geom.B,))
    shape = (geom.B, geom.Hkv, N, geom.D)
    clear = k is None and v is None
    if clear:
        k, v = k_scales.new_empty((2, *shape), dtype=torch.float16).unbind(0)
    else:
        if k is None:
            k = torch.zeros(shape, dtype=torch.float16, device=k_pages.device)
        if v is None:
            v = torch.zeros(shape, dtype=torch.float16, device=k_pages.device)
        _need(k, torch.float16, "k")
        _need(v, torch.float16, "v")
        if k.shape != shape or v.shape != shape:
            raise ValueError(f"k and v must be {list(shape)}")
    _on(device, table, ctx_len, k, v)
    rows = N * geom.D
    _run(load_library().antkv_qpage_load, "antkv_qpage_load", device, geom._c,
         k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), n_pages, page_size, table.data_ptr(), cap, _p(ctx_len), first, N,
         k.data_ptr(), v.data_ptr(), geom.Hkv * rows, rows, geom.D, clear, _stream(k_pages))
    return k, v


def qpage_attn_workspace(geom: Geometry, T: int, device) -> torch.Tensor:
    """A workspace of antkv_qpage_attn_workspace(geom, T) bytes for qpage_attn, for calls that follow each other on one stream with up to
    T rows."""
    nbytes = load_library().antkv_qpage_attn_workspace(geom._c, T)
    if nbytes == 0 and T != 0 and geom.B != 0:
        raise ValueError(f"qpage_attn does not take {T} rows of this geometry")
    return _workspace(nbytes, device)


def qpage_attn(geom: Geometry, q: torch.Tensor, scale: float, q_start: torch.Tensor, ctx_len: torch.Tensor, table: torch.Tensor, k_pages: torch.Tensor,
               v_pages: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor, window: int = 0, n_sink: int = 0, out: torch.Tensor | None = None,
               want_stats: bool = False, workspace: torch.Tensor | None = None):
    """antkv_qpage_attn: page_attn over pools float8_e4m3fn [n_pages,Hkv,page_size,D] with scales fp32 [n_pages,Hkv,page_size/16]."""
    Hq, R = geom.Hq, geom.B
    _rows(q, "q", Hq)
    n_pages, page_size, device = _byte_pools(k_pages, v_pages, k_scales, v_scales, geom.Hkv)
    T, strides, held = q.shape[0], q.stride(), table.shape
    if (q_start.dtype is not _INT or ctx_len.dtype is not _INT or table.dtype is not _INT or q_start.shape != (R + 1,) or ctx_len.shape != (R,) or len(held) != 2
            or held[0] != R or not (q_start.is_contiguous() and ctx_len.is_contiguous() and table.is_contiguous())):
        _ints(q_start, "q_start", (R + 1,))
        _ints(ctx_len, "ctx_len", (R,))
        _table(table, R)
    if out is None:
        out = q.new_empty((T, Hq, 128))
    else:
        _need(out, _HALF, "out")
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    row_max = row_sum = None
    if want_stats:
        row_max, row_sum = torch.empty((2, Hq, T), dtype=torch.float32, device=q.device).unbind(0)
    if workspace is None:
        workspace = _workspace(load_library().antkv_qpage_attn_workspace(geom._c, T), q.device)
    else:
        _need(workspace, torch.uint8, "workspace")
    _on(device, q, q_start, ctx_len, table, out, workspace)
    _run(load_library().antkv_qpage_attn, "antkv_qpage_attn", device, geom._c, q.data_ptr(), strides[0] if T > 1 else 0,
         strides[1] if Hq > 1 else 0, T, q_start.data_ptr(), ctx_len.data_ptr(), table.data_ptr(), held[1],
         k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), n_pages, page_size, float(scale), int(window), int(n_sink),
         out.data_ptr(), _p(row_max), _p(row_sum), workspace.data_ptr(), workspace.numel(), _stream(q))
    return out, row_max, row_sum


# ---- rotary positions ---------------------------------------------------------------------------------------------------

def rope_freqs(rot_dim: int = 128, base: float = 10000.0, factor: float = 1.0, trained_len: float = 0, slow_turns: float = 1.0, fast_turns: float = 4.0,
               device="cuda") -> torch.Tensor:
    """antkv_rope_freqs: radians per position fp64 [rot_dim/2] for rope; base^(-2i/rot_dim), all of them / factor, or with a trained_len
    only those that turn less than fast_turns times within it (wholly from slow_turns down)."""
    freqs = torch.empty(max(int(rot_dim), 0) // 2, dtype=torch.float64, device=device)
    if not freqs.is_cuda:
        raise ValueError("freqs are made on a GPU")
    _run(load_library().antkv_rope_freqs, "antkv_rope_freqs", freqs.get_device(), int(rot_dim), float(base), float(factor), float(trained_len),
         float(slow_turns), float(fast_turns), freqs.data_ptr(), _stream(freqs))
    return freqs


def _rope_rows(x: torch.Tensor, out: torch.Tensor | None, name: str, heads: int, batch: int, packed: bool, device: int):
    """x fp16 [T,heads,D] (packed, or one sequence) or [B,heads,T,D], channels contiguous -> (T, out, address and strides b, t, h of x, of out)."""
    shape, a = x.shape, x.stride()
    if len(a) == 3:
        T, h, d = shape
        fits = packed or batch == 1
    elif len(a) == 4:
        b, h, T, d = shape
        fits = b == batch and not packed
    else:
        fits = False
    if not fits or h != heads or d != 128 or a[-1] != 1 or x.dtype is not _HALF or x.get_device() != device or device < 0:
        if not x.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        if x.dtype is not _HALF:
            raise TypeError(f"{name} must be torch.float16")
        if x.get_device() != device:
            raise ValueError("all tensors must be on the same device")
        raise ValueError(f"{name} must be [T, {heads}, 128] of a packed batch or of one sequence, or [{batch}, {heads}, T, 128], with contiguous channels")
    if out is None:
        out = x.new_empty(shape)
        o = (128 * h, 128) if len(a) == 3 else (128 * T * h, 128 * T, 128)
    else:
        o = out.stride()
        if out is not x and (out.get_device() != device or out.dtype is not _HALF or out.shape != shape or o[-1] != 1):
            raise ValueError(f"{name}_out must be like {name}")
    if len(a) == 3:
        return T, out, x.data_ptr(), 0, a[0], a[1], out.data_ptr(), 0, o[0], o[1]
    return T, out, x.data_ptr(), a[0], a[2], a[1], out.data_ptr(), o[0], o[2], o[1]


_NO_ROWS = None, None, None, 0, 0, 0, None, 0, 0, 0


def rope(geom: Geometry, q: torch.Tensor | None, k: torch.Tensor | None, freqs: torch.Tensor, pos: torch.Tensor | None = None,
         q_start: torch.Tensor | None = None, ctx_len: torch.Tensor | None = None, pos0: int = 0, style: int = 0, amplitude: float = 1.0,
         inverse: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """antkv_rope: q fp16 [T,Hq,D] and k [T,Hkv,D] of a packed batch (with q_start int32 [B+1] and ctx_len int32 [B], as page_map makes them) or of one
    sequence, or [B,Hq,T,D] and [B,Hkv,T,D]; positions pos (int32, [T] or [B,T]) or pos0, pos0 + 1, ..; freqs fp64 [rot_dim/2] (rope_freqs) ->
    (q_out, k_out), made here where they are not given; q_out=q turns q in place.  Rows outside a packed batch's requests are left as they
    are (undefined where the output is made here).  Records no gradient, and refuses rows that ask for one: that of a call is the same call with
    `inverse` the other way round, of the gradients of its outputs."""
    first = k if q is None else q
    if first is None:
        raise ValueError("q or k must be given")
    if (first.requires_grad or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
        raise ValueError("rope records no gradient: call it under torch.no_grad(), and with the other `inverse` for the gradient")
    packed, device, B = q_start is not None, first.get_device(), geom.B
    rot = freqs.shape
    if freqs.dtype is not torch.float64 or len(rot) != 1 or not freqs.is_contiguous():
        _need(freqs, torch.float64, "freqs")
        raise ValueError("freqs must be [rot_dim / 2]")
    T, q_out, q0, qb, qt, qh, qo0, qob, qot, qoh = _NO_ROWS if q is None else _rope_rows(q, q_out, "q", geom.Hq, B, packed, device)
    Tk, k_out, k0, kb, kt, kh, ko0, kob, kot, koh = _NO_ROWS if k is None else _rope_rows(k, k_out, "k", geom.Hkv, B, packed, device)
    if q is None:
        T = Tk
    elif k is not None and (T != Tk or q.dim() != k.dim()):
        raise ValueError("q and k must have the same rows")
    if packed:
        if ctx_len is None:
            raise ValueError("q_start needs ctx_len")
        if (q_start.dtype is not _INT or ctx_len.dtype is not _INT or q_start.shape != (B + 1,) or ctx_len.shape != (B,)
                or not (q_start.is_contiguous() and ctx_len.is_contiguous())):
            _ints(q_start, "q_start", (B + 1,))
            _ints(ctx_len, "ctx_len", (B,))
    if pos is not None:
        _ints(pos, "pos", (T,) if first.dim() == 3 else (B, T))
    _on(device, freqs, q_start, ctx_len, pos)
    _run(load_library().antkv_rope, "antkv_rope", device, geom._c, q0, qb, qt, qh, k0, kb, kt, kh, T, _p(pos), _p(q_start), _p(ctx_len), pos0, freqs.data_ptr(),
         2 * rot[0], style, amplitude, inverse, qo0, qob, qot, qoh, ko0, kob, kot, koh, _stream(first))
    return q_out, k_out
