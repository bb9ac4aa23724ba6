"""Python binding of libnkv, the MI355X (gfx950) NestedKV prefill compression pass.

Argument marshalling only: every step of the pass runs in the HIP kernels behind the C ABI declared in
``include/nkv.h``; the functions here have the same names as the C entry points.  torch is used to own
device memory and streams.  There is no fallback: if ``libnkv.so`` has not been built
(``python -m paper_2605_26678_amd.build``) importing the library raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

from . import build as _build

NKV_OK = 0
NKV_EINVAL, NKV_ESHAPE, NKV_EWORKSPACE, NKV_EHIP, NKV_EUNSUPPORTED, NKV_ESCRATCH = -1, -2, -3, -4, -5, -6
STATIC_SCRATCH_BYTES = 32 << 20
DTYPE_F32, DTYPE_BF16, DTYPE_F16, DTYPE_F8_E4M3 = 0, 1, 2, 3
FLAG_GENERIC_KERNELS = 1
FLAG_TWO_PASS_STABLE = 2
FLAG_DEFER_STABLE = 4
FLAG_NO_UNIT_SUMS = 8
FLAG_BUDGET_PER_HEAD = 16
FLAG_STATS_PER_HEAD = 32
FLAG_VECTOR_SCAN = 128
FLAG_SELECT_PER_HEAD = 64
FLAG_COMPACT_IN_PLACE = 256
PIN = 3.0e38
PAGE_ROWS = 64
PAGES_16BIT, PAGES_FP4 = 0, 1
ROPE_HALVES, ROPE_PAIRS = 0, 1
MAX_BEAMS_OUT = 64

EXPORTS = ("nkv_params_default", "nkv_block_size", "nkv_k0", "nkv_m_safe", "nkv_m_p", "nkv_packed_rows",
           "nkv_workspace_bytes", "nkv_score", "nkv_score_raw", "nkv_budget", "nkv_budget_noalloc", "nkv_select_compact",
           "nkv_decode_workspace_bytes", "nkv_decode_attention", "nkv_page_bytes", "nkv_pages_append", "nkv_pages_load",
           "nkv_pages_read", "nkv_pages_workspace_bytes", "nkv_pages_attention", "nkv_pages_prompt_workspace_bytes", "nkv_pages_prompt_attention", "nkv_pages_copy", "nkv_pages_compact",
           "nkv_beam_workspace_bytes", "nkv_beam_select", "nkv_copy_probe", "nkv_strerror", "nkv_version")
KERNELS = ("scan", "finalize", "budget", "select", "gather", "decode")
PASS_KERNELS = KERNELS[:5]          # the kernels of the compression pass itself


class nkv_params(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("window", C.c_int32), ("block_div", C.c_int32),
                ("block_min", C.c_int32), ("block_max", C.c_int32), ("n_sink", C.c_int32),
                ("gate_mode", C.c_int32), ("surprise_mode", C.c_int32), ("flags", C.c_uint32),
                ("scale_mask", C.c_int32), ("top_frac", C.c_double), ("prior", C.c_double * 3),
                ("beta", C.c_double), ("tau", C.c_double), ("kappa", C.c_double), ("safeguard", C.c_double),
                ("near_tol", C.c_double), ("prof_start", C.c_void_p * 6), ("prof_stop", C.c_void_p * 6),
                ("scan_counters", C.c_void_p)]


class nkv_shape(C.Structure):
    _fields_ = [("L", C.c_int32), ("H", C.c_int32), ("d", C.c_int32), ("dv", C.c_int32), ("dtype", C.c_int32),
                ("n_prompts", C.c_int32), ("cu_seqlens", C.POINTER(C.c_int32)),
                ("key_strides", C.POINTER(C.c_int64)), ("value_strides", C.POINTER(C.c_int64)),
                ("key_layer_offsets", C.POINTER(C.c_int64)), ("value_layer_offsets", C.POINTER(C.c_int64))]


class nkv_pages(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_seqs", C.c_int32), ("H", C.c_int32), ("d", C.c_int32),
                ("dtype", C.c_int32), ("format", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32),
                ("pool", C.c_void_p), ("table", C.c_void_p), ("lens", C.c_void_p)]


class nkv_tokens(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_new", C.c_int32), ("n_q_heads", C.c_int32), ("rot", C.c_int32),
                ("rope_style", C.c_int32), ("n_positions", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("q", C.c_void_p), ("q_out", C.c_void_p), ("k_strides", C.c_int64 * 3),
                ("v_strides", C.c_int64 * 3), ("q_strides", C.c_int64 * 3), ("positions", C.c_void_p),
                ("rope", C.c_void_p)]


class nkv_logit_rules(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("window", C.c_int32), ("cap", C.c_double), ("slopes", C.c_void_p), ("prefix", C.c_void_p)]


class nkv_beams(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_prompts", C.c_int32), ("n_beams", C.c_int32), ("vocab", C.c_int32), ("n_out", C.c_int32),
                ("dtype", C.c_int32), ("strides", C.c_int64 * 2), ("logits", C.c_void_p), ("scores", C.c_void_p)]


_TOKENS_SIZE = C.sizeof(nkv_tokens)
_TOKENS = struct.Struct("Iiiiii4P9q2P")        # nkv_tokens' fields in their order, packed in half the time of a ctypes structure
assert _TOKENS.size == _TOKENS_SIZE
_BEAMS_SIZE = C.sizeof(nkv_beams)
_BEAMS = struct.Struct("I5i2q2P")              # nkv_beams' fields likewise
assert _BEAMS.size == _BEAMS_SIZE


class NkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


_lib = None


def lib() -> C.CDLL:
    """The loaded C-ABI library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        path = _build.library_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with `python -m paper_2605_26678_amd.build`")
        L = C.CDLL(path)
        vp, i64, f64 = C.c_void_p, C.c_int64, C.c_double
        L.nkv_params_default.argtypes = [C.POINTER(nkv_params)]
        L.nkv_block_size.argtypes = [i64, C.POINTER(nkv_params)]
        L.nkv_block_size.restype = i64
        L.nkv_k0.argtypes = [i64, f64]
        L.nkv_k0.restype = i64
        L.nkv_m_safe.argtypes = [i64, f64]
        L.nkv_m_safe.restype = i64
        L.nkv_m_p.argtypes = [i64, f64]
        L.nkv_m_p.restype = i64
        L.nkv_packed_rows.argtypes = [C.POINTER(nkv_shape), C.POINTER(f64), C.POINTER(i64)]
        L.nkv_workspace_bytes.argtypes = [C.POINTER(nkv_shape), C.POINTER(nkv_params), C.POINTER(C.c_size_t)]
        L.nkv_score.argtypes = [vp, C.POINTER(nkv_shape), C.POINTER(nkv_params), vp, vp, C.c_size_t, vp]
        L.nkv_score_raw.argtypes = [vp, C.POINTER(nkv_shape), C.POINTER(nkv_params), vp, vp, C.c_size_t, vp]
        L.nkv_budget.argtypes = [vp, C.POINTER(nkv_shape), C.POINTER(nkv_params), C.POINTER(f64), vp, vp,
                                 C.c_size_t, vp]
        L.nkv_budget_noalloc.argtypes = [vp, C.POINTER(nkv_shape), C.POINTER(nkv_params), C.POINTER(f64), vp, vp]
        L.nkv_select_compact.argtypes = [vp, vp, vp, vp, C.POINTER(nkv_shape), C.POINTER(nkv_params), vp, vp, vp,
                                         vp, i64, vp, vp, C.c_size_t, vp]
        L.nkv_decode_workspace_bytes.argtypes = [C.POINTER(nkv_shape), C.c_int32, i64, C.POINTER(C.c_size_t)]
        L.nkv_decode_attention.argtypes = [vp, vp, vp, vp, i64, C.POINTER(nkv_shape), C.POINTER(nkv_params),
                                           C.c_int32, f64, vp, vp, vp, C.c_size_t, vp]
        L.nkv_page_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
        L.nkv_page_bytes.restype = i64
        L.nkv_pages_append.argtypes = [vp, C.POINTER(nkv_pages), vp]           # nkv_tokens *, by a structure or its bytes
        L.nkv_pages_load.argtypes = [vp, vp, vp, i64, C.POINTER(nkv_pages), vp]
        L.nkv_pages_read.argtypes = [vp, vp, vp, i64, C.POINTER(nkv_pages), vp]
        L.nkv_pages_workspace_bytes.argtypes = [C.POINTER(nkv_pages), C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.nkv_pages_attention.argtypes = [vp, C.POINTER(nkv_pages), C.c_int32, C.c_int32, f64, vp, vp, vp,
                                          C.c_size_t, vp]
        L.nkv_pages_prompt_workspace_bytes.argtypes = [C.POINTER(nkv_pages), C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.nkv_pages_prompt_attention.argtypes = [vp, C.POINTER(nkv_pages), C.POINTER(nkv_logit_rules), C.c_int32, C.c_int32, f64, vp, vp, vp,
                                                 C.c_size_t, vp]
        L.nkv_pages_copy.argtypes = [vp, vp, i64, C.POINTER(nkv_pages), vp]
        L.nkv_pages_compact.argtypes = [vp, vp, i64, C.POINTER(nkv_pages), C.POINTER(nkv_pages), vp]
        L.nkv_beam_workspace_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]      # nkv_beams *, likewise
        L.nkv_beam_select.argtypes = [vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.nkv_copy_probe.argtypes = [vp, vp, C.c_size_t, vp]
        L.nkv_strerror.argtypes = [C.c_int]
        L.nkv_strerror.restype = C.c_char_p
        L.nkv_version.restype = C.c_int
        for name in EXPORTS:
            getattr(L, name)
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().nkv_strerror(int(status)).decode()


def params_default(**overrides) -> nkv_params:
    p = nkv_params()
    rc = lib().nkv_params_default(C.byref(p))
    if rc:
        raise NkvError(rc, "nkv_params_default")
    for k, v in overrides.items():
        if k == "prior":
            p.prior = (C.c_double * 3)(*v)
        else:
            if not hasattr(p, k):
                raise AttributeError(k)
            setattr(p, k, v)
    return p


def block_size(N: int, params: Optional[nkv_params] = None) -> int:
    p = params or params_default()
    return int(lib().nkv_block_size(int(N), C.byref(p)))


def k0(N: int, r: float) -> int:
    return int(lib().nkv_k0(int(N), float(r)))


def m_safe(k0_: int, safeguard: float = 0.20) -> int:
    return int(lib().nkv_m_safe(int(k0_), float(safeguard)))


def m_p(N: int, top_frac: float = 0.10) -> int:
    return int(lib().nkv_m_p(int(N), float(top_frac)))


class Shape:
    """Host-side description of keys[L][H][T][d] / values[L][H][T][dv] holding one or more prompts.
    ``key_strides`` / ``value_strides``: None for the dense layout, else (layer, head, prompt) strides in
    elements as ``nkv_shape`` in nkv.h defines them.  ``key_layers`` / ``value_layers``: None, or one tensor
    (or device address) per layer when every layer has a tensor of its own; the calls are then handed layer
    0's tensor."""

    def __init__(self, L: int, H: int, d: int, dv: int, dtype: int, cu_seqlens: Sequence[int],
                 key_strides: Optional[Sequence[int]] = None, value_strides: Optional[Sequence[int]] = None,
                 key_layers: Optional[Sequence] = None, value_layers: Optional[Sequence] = None):
        self.cu = (C.c_int32 * len(cu_seqlens))(*[int(x) for x in cu_seqlens])
        self.ks = None if key_strides is None else (C.c_int64 * 3)(*[int(x) for x in key_strides])
        self.vs = None if value_strides is None else (C.c_int64 * 3)(*[int(x) for x in value_strides])
        esize = {DTYPE_F32: 4, DTYPE_BF16: 2, DTYPE_F16: 2, DTYPE_F8_E4M3: 1}.get(int(dtype), 1)

        def offsets(layers):
            if layers is None:
                return None
            addr = [int(t) if isinstance(t, int) else int(t.data_ptr()) for t in layers]
            if len(addr) != int(L) or any((a - addr[0]) % esize for a in addr):
                raise ValueError("one tensor per layer, element-aligned")
            return (C.c_int64 * len(addr))(*[(a - addr[0]) // esize for a in addr])

        self.klo, self.vlo = offsets(key_layers), offsets(value_layers)
        self.c = nkv_shape(int(L), int(H), int(d), int(dv), int(dtype), len(cu_seqlens) - 1, self.cu,
                           self.ks, self.vs, self.klo, self.vlo)
        self.L, self.H, self.d, self.dv, self.dtype = int(L), int(H), int(d), int(dv), int(dtype)
        self.n_prompts = len(cu_seqlens) - 1
        self.T = int(cu_seqlens[-1])
        self.cu_seqlens = [int(x) for x in cu_seqlens]

    @property
    def n_units(self) -> int:
        return self.n_prompts * self.L * self.H


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


_current_stream = None


def _find_current_stream():
    """The current device's current stream as a number.  torch's own short cut to it where there is one: a Stream object is 3 us of a
    call's 7."""
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    torch.cuda.current_stream()                          # (initialises the device)
    if raw is None or device is None:
        return lambda: int(torch.cuda.current_stream().cuda_stream)
    return lambda: raw(device())


def _stream(stream) -> int:
    if stream is None:
        global _current_stream
        if _current_stream is None:
            _current_stream = _find_current_stream()
        return _current_stream()
    return int(getattr(stream, "cuda_stream", stream))


def packed_rows(shape: Shape, r_per_prompt: Sequence[float]) -> int:
    r = (C.c_double * shape.n_prompts)(*[float(x) for x in r_per_prompt])
    out = C.c_int64(0)
    rc = lib().nkv_packed_rows(C.byref(shape.c), r, C.byref(out))
    if rc:
        raise NkvError(rc, "nkv_packed_rows")
    return int(out.value)


def workspace_bytes(shape: Shape, params: Optional[nkv_params] = None) -> int:
    p = params or params_default()
    out = C.c_size_t(0)
    rc = lib().nkv_workspace_bytes(C.byref(shape.c), C.byref(p), C.byref(out))
    if rc:
        raise NkvError(rc, "nkv_workspace_bytes")
    return int(out.value)


def score(keys, shape: Shape, params: nkv_params, scores, ws, stream=None) -> None:
    """keys [L,H,T,d] (device) -> scores [L,H,T] fp32 (device), enqueued on ``stream``."""
    rc = lib().nkv_score(_ptr(keys), C.byref(shape.c), C.byref(params), _ptr(scores), _ptr(ws),
                         0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_score")


def score_raw(keys, shape: Shape, params: nkv_params, a_raw, ws, stream=None) -> None:
    """keys -> a_raw [3,L,H,T] fp32: the per-scale anomalies before normalisation."""
    rc = lib().nkv_score_raw(_ptr(keys), C.byref(shape.c), C.byref(params), _ptr(a_raw), _ptr(ws),
                             0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_score_raw")


def budget(scores, shape: Shape, params: nkv_params, r_per_prompt: Sequence[float], k_per_head, ws=None,
           stream=None) -> None:
    """scores [L,H,T] -> k_per_head [P,L,H] int32."""
    r = (C.c_double * shape.n_prompts)(*[float(x) for x in r_per_prompt])
    rc = lib().nkv_budget(_ptr(scores), C.byref(shape.c), C.byref(params), r, _ptr(k_per_head), _ptr(ws),
                          0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_budget")


def budget_noalloc(scores, shape: Shape, params: nkv_params, r_per_prompt: Sequence[float], k_per_head,
                   stream=None) -> None:
    """``budget`` on the library's own static scratch array (no workspace argument, nothing allocated)."""
    r = (C.c_double * shape.n_prompts)(*[float(x) for x in r_per_prompt])
    rc = lib().nkv_budget_noalloc(_ptr(scores), C.byref(shape.c), C.byref(params), r, _ptr(k_per_head),
                                  _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_budget_noalloc")


def select_compact(keys, values, scores, k_per_head, shape: Shape, params: nkv_params, packed_k, packed_v,
                   kept_idx, head_off, row_capacity: int, near_threshold_count=None, ws=None, stream=None) -> None:
    """Top-B_h selection, ordered compaction and K/V gather; see ``nkv_select_compact`` in nkv.h."""
    rc = lib().nkv_select_compact(_ptr(keys), _ptr(values), _ptr(scores), _ptr(k_per_head), C.byref(shape.c),
                                  C.byref(params), _ptr(packed_k), _ptr(packed_v), _ptr(kept_idx), _ptr(head_off),
                                  int(row_capacity), _ptr(near_threshold_count), _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_select_compact")


def decode_workspace_bytes(shape: Shape, n_q_heads: int, rows: int) -> int:
    out = C.c_size_t(0)
    rc = lib().nkv_decode_workspace_bytes(C.byref(shape.c), int(n_q_heads), int(rows), C.byref(out))
    if rc:
        raise NkvError(rc, "nkv_decode_workspace_bytes")
    return int(out.value)


def decode_attention(q, packed_k, packed_v, head_off, rows: int, shape: Shape, params: nkv_params, n_q_heads: int,
                     scale: float, out, lse=None, ws=None, stream=None) -> None:
    """One new token's attention over the compressed cache: q [P,L,Hq,d] -> out [P,L,Hq,dv] fp32 (and lse
    [P,L,Hq]); see ``nkv_decode_attention`` in nkv.h."""
    rc = lib().nkv_decode_attention(_ptr(q), _ptr(packed_k), _ptr(packed_v), _ptr(head_off), int(rows),
                                    C.byref(shape.c), C.byref(params), int(n_q_heads), float(scale), _ptr(out),
                                    _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_decode_attention")


class Pages:
    """A paged cache as ``nkv_pages`` in nkv.h describes it: ``pool`` (uint8, n_pages * page_bytes), ``table`` int32
    [n_seqs * H, max_pages], ``lens`` int32 [n_seqs * H], all on the device and owned by the caller."""

    def __init__(self, n_seqs: int, H: int, d: int, dtype: int, format: int, pool, table, lens):
        import torch
        size = page_bytes(d, dtype, format)
        if size < 0:
            raise NkvError(NKV_EUNSUPPORTED, "nkv_page_bytes")
        nbytes = pool.numel() * pool.element_size()
        if table.dtype != torch.int32 or lens.dtype != torch.int32 or table.shape[0] != n_seqs * H or \
                table.dim() != 2 or lens.numel() != n_seqs * H or nbytes < size:
            raise ValueError("table is int32 [n_seqs * H, max_pages], lens int32 [n_seqs * H], the pool a page or more")
        if not (pool.is_contiguous() and table.is_contiguous() and lens.is_contiguous()):
            raise ValueError("pool, table and lens are contiguous")
        if not pool.device == table.device == lens.device:
            raise ValueError("pool, table and lens are on one device")
        self.pool, self.table, self.lens = pool, table, lens
        self.n_seqs, self.H, self.d, self.dtype, self.format = int(n_seqs), int(H), int(d), int(dtype), int(format)
        self.units = self.n_seqs * self.H
        self.index = pool.get_device()                   # of the GPU; -1: the CPU
        self.torch_dtype, self.torch_f32, self.torch_i32, self.torch_i64 = _torch_dtype(dtype), torch.float32, torch.int32, torch.int64
        self.c = nkv_pages(C.sizeof(nkv_pages), int(n_seqs), int(H), int(d), int(dtype), int(format), nbytes // size,
                           int(table.shape[1]), _ptr(pool), _ptr(table), _ptr(lens))
        self.ref = C.byref(self.c)


def page_bytes(d: int, dtype: int, format: int) -> int:
    """Bytes of a page of 64 rows; -1 for rows that are not supported."""
    return int(lib().nkv_page_bytes(int(d), int(dtype), int(format)))


def rope_table(n_positions: int, rot: int, base: float = 10000.0, device="cuda"):
    """Cosines and sines [n_positions, 2, rot / 2] of position * base^(-2 i / rot), angles in 64 bits."""
    import torch
    f = dict(dtype=torch.float64, device=device)
    angle = torch.arange(n_positions, **f)[:, None] * base ** (-torch.arange(0, rot, 2, **f) / rot)
    return torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()


def _torch_dtype(dtype: int):
    import torch
    return {DTYPE_F32: torch.float32, DTYPE_BF16: torch.bfloat16, DTYPE_F16: torch.float16}.get(int(dtype))


def _elsewhere(t, what: str, pages: Pages) -> ValueError:
    return ValueError(f"{what} is on device {t.device}, and the pages are on {pages.pool.device}")


def _check_gpu(pages: Pages) -> None:
    """What ends a call's checks: tensors are where the pages are, and those are not on the CPU."""
    if pages.index < 0:
        raise ValueError("the pages are not on a GPU")


def _check_rows(t, what: str, pages: Pages, shape) -> None:
    """Rows that a call reads or writes: their type, their shape, and that they are dense."""
    if t.dtype is not pages.torch_dtype:
        raise ValueError(f"{what} is {t.dtype}, and the pages' rows are {pages.torch_dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} is dense {list(shape)}")
    if t.get_device() != pages.index:
        raise _elsewhere(t, what, pages)


def _check_dense(t, what: str, pages: Pages, dtype, numbers: int) -> None:
    """A buffer that a call indexes by itself: its type, that it is contiguous, and how much it holds."""
    if t.dtype is not dtype or not t.is_contiguous() or t.numel() < numbers:
        raise ValueError(f"{what} is contiguous {dtype} of {numbers} numbers, not {t.dtype} {list(t.shape)} by strides {list(t.stride())}")
    if t.get_device() != pages.index:
        raise _elsewhere(t, what, pages)


def _strides(t, what: str, pages: Pages, given, shape):
    """Strides of a new token's rows [n_seqs, n, heads, d] (0 along a dim of one); their type, shape (`given`) and device are checked."""
    if t.dtype is not pages.torch_dtype or given != shape:
        raise ValueError(f"{what} is {pages.torch_dtype} {list(shape)}, not {t.dtype} {list(given)}")
    s, n, h, e = t.stride()
    if e != 1:
        raise ValueError(f"{what}: a row's dims lie next to each other")
    if t.get_device() != pages.index:
        raise _elsewhere(t, what, pages)
    return s if shape[0] > 1 else 0, n if shape[1] > 1 else 0, h if shape[2] > 1 else 0


def pages_append(k, v, pages: Pages, positions=None, rope=None, rope_style: int = ROPE_HALVES, q=None, q_out=None,
                 stream=None) -> None:
    """New tokens' k, v [n_seqs, n, H, d] (any strides but the last dim's) to the last n rows of the pages, k rotated
    by ``rope`` [n_positions, 2, rot / 2] at ``positions`` int32 [n_seqs, n] on the way; q [n_seqs, n, Hq, d] rotated
    into q_out; see ``nkv_pages_append`` in nkv.h."""
    given = k.shape                                      # (a tensor's shape, device or type is some 0.1 us of a call's 7 each time)
    S, n, d = pages.n_seqs, given[1], pages.d
    shape = (S, n, pages.H, d)
    ks, vs = _strides(k, "k", pages, given, shape), _strides(v, "v", pages, v.shape, shape)
    Hq, qs, q_at, out_at = 0, (0, 0, 0), 0, 0
    if q is not None:
        if q_out is None:
            raise ValueError("q and q_out are given together")
        given = q.shape
        Hq = given[2]
        shape = (S, n, Hq, d)
        qs, q_at, out_at = _strides(q, "q", pages, given, shape), q.data_ptr(), q_out.data_ptr()
        _check_rows(q_out, "q_out", pages, shape)
    elif q_out is not None:
        raise ValueError("q and q_out are given together")
    rot = n_positions = rope_at = pos_at = 0
    if rope is not None:
        given = rope.shape
        if rope.dtype is not pages.torch_f32 or len(given) != 3 or given[1] != 2 or not rope.is_contiguous():
            raise ValueError("rope is fp32 [n_positions, 2, rot / 2], contiguous")
        if rope.get_device() != pages.index:
            raise _elsewhere(rope, "rope", pages)
        rot, n_positions, rope_at = 2 * given[2], given[0], rope.data_ptr()
    if positions is not None:
        if positions.dtype is not pages.torch_i32 or positions.numel() != S * n or not positions.is_contiguous():
            raise ValueError("positions is int32 [n_seqs, n], contiguous")
        if positions.get_device() != pages.index:
            raise _elsewhere(positions, "positions", pages)
        pos_at = positions.data_ptr()
    _check_gpu(pages)
    tokens = _TOKENS.pack(_TOKENS_SIZE, n, Hq, rot, rope_style, n_positions, k.data_ptr(), v.data_ptr(), q_at, out_at,
                          *ks, *vs, *qs, pos_at, rope_at)
    rc = lib().nkv_pages_append(tokens, pages.ref, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_append")


def _check_packed(packed_k, packed_v, head_off, rows: int, pages: Pages) -> None:
    at, dtype, numbers = pages.index, pages.torch_dtype, rows * pages.d
    if packed_k.dtype is dtype and packed_k.is_contiguous() and packed_k.numel() >= numbers and packed_k.get_device() == at and \
            packed_v.dtype is dtype and packed_v.is_contiguous() and packed_v.numel() >= numbers and packed_v.get_device() == at and \
            head_off.dtype is pages.torch_i64 and head_off.is_contiguous() and head_off.numel() > pages.units and \
            head_off.get_device() == at >= 0:
        return                                           # (the same one after the other takes a microsecond more)
    _check_dense(packed_k, "packed_k", pages, dtype, numbers)
    _check_dense(packed_v, "packed_v", pages, dtype, numbers)
    _check_dense(head_off, "head_off", pages, pages.torch_i64, pages.units + 1)
    _check_gpu(pages)


def pages_load(packed_k, packed_v, head_off, rows: int, pages: Pages, stream=None) -> None:
    """Packed rows [rows, d] (as ``select_compact`` leaves them) to the end of every unit's pages."""
    rows = int(rows)
    _check_packed(packed_k, packed_v, head_off, rows, pages)
    rc = lib().nkv_pages_load(packed_k.data_ptr(), packed_v.data_ptr(), head_off.data_ptr(), rows, pages.ref, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_load")


def pages_read(packed_k, packed_v, head_off, rows: int, pages: Pages, stream=None) -> None:
    """The last head_off[u + 1] - head_off[u] rows of every unit to packed rows [rows, d]."""
    rows = int(rows)
    _check_packed(packed_k, packed_v, head_off, rows, pages)
    rc = lib().nkv_pages_read(packed_k.data_ptr(), packed_v.data_ptr(), head_off.data_ptr(), rows, pages.ref, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_read")


def pages_workspace_bytes(pages: Pages, n_q_heads: int, n_new: int = 1) -> int:
    """Scratch of ``pages_attention``: it grows with n_new times the query heads, see nkv.h; hand over many tokens some at a time."""
    out = C.c_size_t(0)
    rc = lib().nkv_pages_workspace_bytes(pages.ref, int(n_q_heads), int(n_new), C.byref(out))
    if rc:
        raise NkvError(rc, "nkv_pages_workspace_bytes")
    return int(out.value)


def pages_attention(q, pages: Pages, n_q_heads: int, n_new: int, scale: float, out, lse=None, ws=None,
                    stream=None) -> None:
    """The last n_new tokens' attention over the pages: q [n_seqs, n_new, Hq, d] -> out fp32 of that shape (and lse
    [n_seqs, n_new, Hq]); see ``nkv_pages_attention`` in nkv.h."""
    _check_rows(q, "q", pages, (pages.n_seqs, n_new, n_q_heads, pages.d))
    columns = pages.n_seqs * n_new * n_q_heads
    _check_dense(out, "out", pages, pages.torch_f32, columns * pages.d)
    if lse is not None:
        _check_dense(lse, "lse", pages, pages.torch_f32, columns)
    ws_at = ws_bytes = 0
    if ws is not None:
        if not ws.is_contiguous():
            raise ValueError("ws is contiguous")
        if ws.get_device() != pages.index:
            raise _elsewhere(ws, "ws", pages)
        ws_at, ws_bytes = ws.data_ptr(), ws.nbytes
    _check_gpu(pages)
    rc = lib().nkv_pages_attention(q.data_ptr(), pages.ref, int(n_q_heads), int(n_new), float(scale), out.data_ptr(),
                                   0 if lse is None else lse.data_ptr(), ws_at, ws_bytes, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_attention")


class LogitRules:
    """Rules for the logits of ``pages_prompt_attention``, as ``nkv_logit_rules`` in nkv.h describes them: ``cap`` (0: none), ``window`` (0: none), ``slopes``
    fp32 [n_q_heads] and ``prefix`` int32 [n_seqs] on the device, or None."""

    def __init__(self, cap: float = 0.0, window: int = 0, slopes=None, prefix=None):
        import torch
        for t, what, dtype in ((slopes, "slopes", torch.float32), (prefix, "prefix", torch.int32)):
            if t is not None and (t.dtype is not dtype or t.dim() != 1 or not t.is_contiguous()):
                raise ValueError(f"{what} is contiguous {dtype} of one dim")
        if not cap >= 0.0 or window < 0 or int(window) >= 1 << 31:           # (ctypes cuts a longer number off)
            raise ValueError("cap and window are not negative, and a window is of 31 bits")
        self.cap, self.window, self.slopes, self.prefix = float(cap), int(window), slopes, prefix
        self.c = nkv_logit_rules(C.sizeof(nkv_logit_rules), self.window, self.cap, _ptr(slopes), _ptr(prefix))
        self.ref = C.byref(self.c)


def pages_prompt_workspace_bytes(pages: Pages, n_q_heads: int, n_new: int) -> int:
    """Scratch of ``pages_prompt_attention``; 0 where it needs none."""
    out = C.c_size_t(0)
    rc = lib().nkv_pages_prompt_workspace_bytes(pages.ref, int(n_q_heads), int(n_new), C.byref(out))
    if rc:
        raise NkvError(rc, "nkv_pages_prompt_workspace_bytes")
    return int(out.value)


def pages_prompt_attention(q, pages: Pages, n_q_heads: int, n_new: int, scale: float, out, lse=None, ws=None, rules: Optional[LogitRules] = None,
                           stream=None) -> None:
    """The last n_new tokens' attention over the pages, a prompt's chunk or single tokens, by ``rules``: q [n_seqs, n_new, Hq, d] -> out of that shape and type
    (and lse fp32 [n_seqs, n_new, Hq]); see ``nkv_pages_prompt_attention`` in nkv.h."""
    shape = (pages.n_seqs, n_new, n_q_heads, pages.d)
    _check_rows(q, "q", pages, shape)
    _check_rows(out, "out", pages, shape)
    if lse is not None:
        _check_dense(lse, "lse", pages, pages.torch_f32, pages.n_seqs * n_new * n_q_heads)
    rules_at = None
    if rules is not None:
        rules_at = rules.ref
        if rules.slopes is not None:
            _check_dense(rules.slopes, "slopes", pages, pages.torch_f32, n_q_heads)
        if rules.prefix is not None:
            _check_dense(rules.prefix, "prefix", pages, pages.torch_i32, pages.n_seqs)
    ws_at = ws_bytes = 0
    if ws is not None:
        if not ws.is_contiguous():
            raise ValueError("ws is contiguous")
        if ws.get_device() != pages.index:
            raise _elsewhere(ws, "ws", pages)
        ws_at, ws_bytes = ws.data_ptr(), ws.nbytes
    _check_gpu(pages)
    rc = lib().nkv_pages_prompt_attention(q.data_ptr(), pages.ref, rules_at, int(n_q_heads), int(n_new), float(scale), out.data_ptr(),
                                          0 if lse is None else lse.data_ptr(), ws_at, ws_bytes, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_prompt_attention")


def pages_copy(src, dst, pages: Pages, stream=None) -> None:
    """Page src[i] to page dst[i] of the pool, src and dst int32 of the same length; see ``nkv_pages_copy`` in nkv.h."""
    n = src.numel()
    if dst.numel() != n:
        raise ValueError(f"src has {n} pages and dst {dst.numel()}")
    at, i32 = pages.index, pages.torch_i32
    if not (src.dtype is i32 and src.is_contiguous() and src.get_device() == at and dst.dtype is i32 and dst.is_contiguous() and dst.get_device() == at >= 0):
        _check_dense(src, "src", pages, i32, n)
        _check_dense(dst, "dst", pages, i32, n)
        _check_gpu(pages)
    rc = lib().nkv_pages_copy(src.data_ptr(), dst.data_ptr(), n, pages.ref, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_copy")


def pages_compact(kept_idx, head_off, rows: int, old: Pages, pages: Pages, stream=None) -> None:
    """Rows kept_idx[head_off[u] .. head_off[u + 1] - 1] (int32, numbers within the unit) of every unit of ``old`` to the front of the unit
    in ``pages``, which has pages of its own; see ``nkv_pages_compact`` in nkv.h."""
    rows = int(rows)
    if old.index != pages.index:
        raise _elsewhere(old.pool, "old", pages)
    _check_dense(kept_idx, "kept_idx", pages, pages.torch_i32, rows)
    _check_dense(head_off, "head_off", pages, pages.torch_i64, pages.units + 1)
    _check_gpu(pages)
    rc = lib().nkv_pages_compact(kept_idx.data_ptr(), head_off.data_ptr(), rows, old.ref, pages.ref, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_pages_compact")


def beam_workspace_bytes(n_prompts: int, n_beams: int, vocab: int, n_out: int) -> int:
    """Scratch of ``beam_select``."""
    out = C.c_size_t(0)
    some = 256                                           # (an address that is not used)
    rc = lib().nkv_beam_workspace_bytes(_BEAMS.pack(_BEAMS_SIZE, n_prompts, n_beams, vocab, n_out, DTYPE_F32, 0, 0, some, some), C.byref(out))
    if rc:
        raise NkvError(rc, "nkv_beam_workspace_bytes")
    return int(out.value)


_beam_types = None


def _find_beam_types():
    import torch
    return {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}, torch.float32, torch.int32


def _check_beam(t, what: str, kind, shape, logits) -> None:
    if t.dtype is not kind or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} is dense {kind} {list(shape)}, not {t.dtype} {list(t.shape)}")
    if t.get_device() != logits.get_device():
        raise ValueError(f"{what} is on device {t.device}, and the logits are on {logits.device}")


def beam_select(logits, scores, out_scores, out_beams, out_tokens, ws, stream=None) -> None:
    """The best candidates of every prompt: logits [P, B, V] of fp32, bf16 or fp16 (any strides but the last dim's), scores fp32 [P, B] ->
    out_scores fp32, out_beams, out_tokens int32 [P, n_out], largest first; see ``nkv_beam_select`` in nkv.h."""
    global _beam_types
    if _beam_types is None:
        _beam_types = _find_beam_types()
    codes, f32, i32 = _beam_types
    dtype, given, strides = codes.get(logits.dtype), logits.shape, logits.stride()
    if dtype is None or len(given) != 3 or strides[2] != 1 and given[2] > 1:
        raise ValueError("logits is fp32, bf16 or fp16 [prompts, beams, vocabulary], a beam's logits next to each other")
    P, B, V = given
    shape, at = out_scores.shape, logits.get_device()
    if len(shape) != 2 or shape[0] != P:
        raise ValueError(f"out_scores is [{P}, n_out]")
    _check_beam(scores, "scores", f32, (P, B), logits)
    _check_beam(out_scores, "out_scores", f32, shape, logits)
    _check_beam(out_beams, "out_beams", i32, shape, logits)
    _check_beam(out_tokens, "out_tokens", i32, shape, logits)
    if not ws.is_contiguous() or ws.get_device() != at:
        raise ValueError("ws is contiguous and on the logits' device")
    if at < 0:
        raise ValueError("the logits are not on a GPU")
    rc = lib().nkv_beam_select(_BEAMS.pack(_BEAMS_SIZE, P, B, V, shape[1], dtype, strides[0], strides[1], logits.data_ptr(), scores.data_ptr()),
                               out_scores.data_ptr(), out_beams.data_ptr(), out_tokens.data_ptr(), ws.data_ptr(), ws.nbytes, _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_beam_select")


def copy_probe(dst, src, stream=None) -> None:
    """Plain device copy src -> dst (same byte size), the bandwidth yardstick; dst None: loads only."""
    rc = lib().nkv_copy_probe(_ptr(dst), _ptr(src), src.numel() * src.element_size(), _stream(stream))
    if rc:
        raise NkvError(rc, "nkv_copy_probe")


_hip = None


def _hiprt() -> C.CDLL:
    global _hip
    if _hip is None:
        h = C.CDLL("libamdhip64.so")
        h.hipEventCreate.argtypes = [C.POINTER(C.c_void_p)]
        h.hipEventDestroy.argtypes = [C.c_void_p]
        h.hipEventRecord.argtypes = [C.c_void_p, C.c_void_p]
        h.hipEventSynchronize.argtypes = [C.c_void_p]
        h.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
        _hip = h
    return _hip


class HipEvent:
    """A raw hipEvent_t, recorded by the library (kernel timing) or by the caller on a given stream."""

    def __init__(self):
        self.handle = C.c_void_p()
        rc = _hiprt().hipEventCreate(C.byref(self.handle))
        if rc:
            raise RuntimeError(f"hipEventCreate failed: {rc}")

    def record(self, stream=None) -> None:
        rc = _hiprt().hipEventRecord(self.handle, _stream(stream))
        if rc:
            raise RuntimeError(f"hipEventRecord failed: {rc}")

    def synchronize(self) -> None:
        _hiprt().hipEventSynchronize(self.handle)

    def elapsed_ms(self, later: "HipEvent") -> float:
        ms = C.c_float(0)
        rc = _hiprt().hipEventElapsedTime(C.byref(ms), self.handle, later.handle)
        if rc:
            raise RuntimeError(f"hipEventElapsedTime failed: {rc}")
        return float(ms.value)

    def __del__(self):
        try:
            if self.handle:
                _hiprt().hipEventDestroy(self.handle)
        except Exception:
            pass


def with_kernel_timers(params: nkv_params, timers: dict) -> nkv_params:
    """A copy of ``params`` that asks the library to record ``timers[name] = (start, stop)`` HipEvents around
    the launch of the named kernel (names in KERNELS)."""
    q = nkv_params.from_buffer_copy(params)
    for name, (a, b) in timers.items():
        k = KERNELS.index(name)
        q.prof_start[k] = a.handle
        q.prof_stop[k] = b.handle
    return q


@dataclass
class Compressed:
    scores: "object"        # [L,H,T] fp32
    k_per_head: "object"    # [P,L,H] int32
    head_off: "object"      # [P*L*H+1] int64
    kept_idx: "object"      # [rows] int32
    packed_k: "object"      # [rows,d]
    packed_v: "object"      # [rows,dv]
    near_count: "object"    # [1] int64


class Compressor:
    """Owns the device buffers of one workload shape and runs the three calls back to back."""

    def __init__(self, shape: Shape, r_per_prompt: Sequence[float], params: Optional[nkv_params] = None,
                 device="cuda:0", kv_dtype=None):
        import torch
        self.torch = torch
        self.shape, self.params = shape, params or params_default()
        self.r = [float(x) for x in r_per_prompt]
        self.rows = packed_rows(shape, self.r)
        dev = torch.device(device)
        kv_dtype = kv_dtype or {DTYPE_F32: torch.float32, DTYPE_BF16: torch.bfloat16, DTYPE_F16: torch.float16,
                                DTYPE_F8_E4M3: torch.float8_e4m3fn}[shape.dtype]
        self.ws = torch.empty(max(workspace_bytes(shape, self.params), 256), dtype=torch.uint8, device=dev)
        self.scores = torch.empty(shape.L, shape.H, shape.T, dtype=torch.float32, device=dev)
        self.k_per_head = torch.empty(shape.n_prompts, shape.L, shape.H, dtype=torch.int32, device=dev)
        self.head_off = torch.empty(shape.n_units + 1, dtype=torch.int64, device=dev)
        self.kept_idx = torch.empty(max(self.rows, 1), dtype=torch.int32, device=dev)
        self.packed_k = torch.empty(max(self.rows, 1), shape.d, dtype=kv_dtype, device=dev)
        self.packed_v = torch.empty(max(self.rows, 1), shape.dv, dtype=kv_dtype, device=dev)
        self.near = torch.zeros(1, dtype=torch.int64, device=dev)

    def run(self, keys, values, stream=None) -> Compressed:
        score(keys, self.shape, self.params, self.scores, self.ws, stream)
        budget(self.scores, self.shape, self.params, self.r, self.k_per_head, self.ws, stream)
        select_compact(keys, values, self.scores, self.k_per_head, self.shape, self.params, self.packed_k,
                       self.packed_v, self.kept_idx, self.head_off, self.rows, self.near, self.ws, stream)
        return Compressed(self.scores, self.k_per_head, self.head_off, self.kept_idx[:self.rows],
                          self.packed_k[:self.rows], self.packed_v[:self.rows], self.near)


class PagedCache:
    """Owns a paged cache's pool, table and lengths and hands out its pages, on the host: ``pages`` is what the calls
    take.  ``lens`` (device) is the program's to write; ``reserve`` only sees to it that there are pages: where lengths have gone back
    below rows that sequences share, ``fork`` gives each its own before the next append.  ``layers`` gives a ``Pages`` for every
    layer where the sequences are (prompt, layer).  ``reserve``, ``release``, ``fork`` and ``compact`` write tables
    and lengths where they lie, so recorded graphs go by them, in the current stream's order: that of the calls on the pages."""

    def __init__(self, n_seqs: int, H: int, d: int, dtype: int, format: int, n_pages: int, max_rows: int,
                 device="cuda:0"):
        import torch
        self.n_seqs, self.H = int(n_seqs), int(H)
        size = page_bytes(d, dtype, format)
        if size < 0:
            raise NkvError(NKV_EUNSUPPORTED, "nkv_page_bytes")
        self.pool = torch.zeros(n_pages, size, dtype=torch.uint8, device=device)
        width = max(1, (int(max_rows) + PAGE_ROWS - 1) // PAGE_ROWS)
        self.table = torch.full((n_seqs * H, width), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(n_seqs * H, dtype=torch.int32, device=device)
        self.pages = Pages(n_seqs, H, d, dtype, format, self.pool, self.table, self.lens)
        self._free = list(range(int(n_pages) - 1, -1, -1))
        self._users = [0] * int(n_pages)                 # units that hold a page
        self._held = [[] for _ in range(n_seqs * H)]
        self._layers, self.layer_table, self.layer_lens = [], None, None

    def layers(self, n_layers: int) -> list:
        """A ``Pages`` for every layer, for calls layer by layer; sequence p * n_layers + l is prompt p in layer l, as the
        units of a pass over several layers are numbered.  A layer's units do not lie side by side in ``table`` and ``lens``, so
        the layers have copies: ``layer_table`` [n_layers, prompts * H, ...], which follows ``table``, and ``layer_lens``
        [n_layers, prompts * H], which begins as ``lens`` is at the first call and is the program's to write from then on, beside
        ``lens``, by which ``pages`` goes (``release`` clears both)."""
        if n_layers < 1 or self.n_seqs % n_layers or self._layers and len(self._layers) != n_layers:
            raise ValueError(f"{self.n_seqs} sequences in {n_layers} layers, the same number at every call")
        if not self._layers:
            self.layer_table, self.layer_lens = self._by_layer(self.table, n_layers), self._by_layer(self.lens, n_layers)
            p = self.pages
            self._layers = [Pages(self.n_seqs // n_layers, p.H, p.d, p.dtype, p.format, self.pool, t, n)
                            for t, n in zip(self.layer_table, self.layer_lens)]
        return list(self._layers)

    def _by_layer(self, x, n_layers: int):
        """[(prompt, layer, head), ...] as a dense copy [layer, (prompt, head), ...]."""
        import torch
        return x.unflatten(0, (self.n_seqs // n_layers, n_layers, self.H)).transpose(0, 1).flatten(1, 2).clone(memory_format=torch.contiguous_format)

    def _by_unit(self, x):
        """The way back: [layer, (prompt, head)] as [(prompt, layer, head)]."""
        return x.view(len(self._layers), -1, self.H).transpose(0, 1).flatten()

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def reserve(self, rows: Sequence[int]) -> None:
        """Pages for that many rows of every unit (as many as it has, if that is more): all of them or, when the pool has
        too few or a unit's row of the table is too short, none."""
        rows = [int(x) for x in rows]
        if len(rows) != len(self._held):
            raise ValueError("one number of rows per unit")
        more = [max(0, (n + PAGE_ROWS - 1) // PAGE_ROWS - len(h)) for n, h in zip(rows, self._held)]
        if max(m + len(h) for m, h in zip(more, self._held)) > self.table.shape[1]:
            raise ValueError(f"a unit holds {self.table.shape[1] * PAGE_ROWS} rows")
        if sum(more) > len(self._free):
            raise MemoryError(f"{sum(more)} pages are wanted and {len(self._free)} free")
        for h, m in zip(self._held, more):
            h.extend(self._new() for _ in range(m))
        if any(more):
            self._write()

    def release(self, seq: int) -> None:
        """Gives a sequence's pages back; its lengths become 0."""
        if not 0 <= seq < self.n_seqs:
            raise IndexError(f"sequence {seq} of {self.n_seqs}")
        for u in range(seq * self.H, (seq + 1) * self.H):
            self._drop(self._held[u])
            self._held[u] = []
        self.lens[seq * self.H:(seq + 1) * self.H] = 0
        if self._layers:
            p, l = divmod(seq, len(self._layers))
            self.layer_lens[l, p * self.H:(p + 1) * self.H] = 0
        self._write()

    def _new(self) -> int:
        page = self._free.pop()
        self._users[page] = 1
        return page

    def _drop(self, pages) -> None:
        for page in reversed(pages):
            self._users[page] -= 1
            if not self._users[page]:
                self._free.append(page)

    def fork(self, parents: Sequence[int], rows: Sequence[int]) -> None:
        """Every sequence s goes on from what sequence parents[s] holds (itself, where it is s), as the beams of a search do that
        ``beam_select`` chose; rows: how many every unit holds now.  Full pages are shared from then on.  One that is not full stays
        with one of a parent's sequences (the parent itself, if it goes on), as do pages reserved behind it, and the others get copies of it; so do all where
        it is one of another unit's full pages.  That is how rows go back that were there at an earlier fork (rejected tokens): lengths as they are
        to be, and a fork with those rows, each sequence its own parent or another's, before anything is appended.
        Lengths follow.  With too few pages nothing changes."""
        import torch
        parents, rows = [int(x) for x in parents], [int(x) for x in rows]
        if len(parents) != self.n_seqs or len(rows) != len(self._held) or any(not 0 <= p < self.n_seqs for p in parents):
            raise ValueError("one parent, a sequence's number, per sequence, and one number of rows per unit")
        if any(n < 0 or n > PAGE_ROWS * len(h) for n, h in zip(rows, self._held)):
            raise ValueError("a unit holds no more rows than its pages do")
        n_layers = len(self._layers) or 1
        if any(p % n_layers != s % n_layers for s, p in enumerate(parents)):
            raise ValueError("a sequence goes on from one of its own layer")
        if parents == list(range(self.n_seqs)) and not any(self._users[page] > 1 for n, h in zip(rows, self._held) for page in h[n // PAGE_ROWS:]):
            return
        heir = {}                                        # of a parent, the sequence that keeps its pages: itself before others
        for s, p in enumerate(parents):
            if p not in heir or p == s:
                heir[p] = s
        held, users = [], [0] * len(self._users)
        for p in parents:
            for v in range(p * self.H, (p + 1) * self.H):
                held.append(self._held[v][:rows[v] // PAGE_ROWS])
                for page in held[-1]:
                    users[page] += 1
        # A page that is written on has one user.  Where rows went back it may be another unit's full page, or two heirs' last one.
        units = [(s * self.H + h, p * self.H + h) for keeps in (True, False) for s, p in enumerate(parents) if (heir[p] == s) == keeps for h in range(self.H)]
        copies = []                                      # (unit, its page's number in the unit, page)
        for u, v in units:
            if rows[v] % PAGE_ROWS:
                full = rows[v] // PAGE_ROWS
                page = self._held[v][full]
                held[u].append(page)
                if users[page]:
                    copies.append((u, full, page))
                users[page] = max(users[page], 1)
        for u, v in units[:len(heir) * self.H]:          # in reserve behind it
            for page in self._held[v][-(-rows[v] // PAGE_ROWS):]:
                if not users[page]:
                    held[u].append(page)
                    users[page] = 1
        copies.sort()
        free = self._free + [page for page, n in enumerate(self._users) if n and not users[page]]
        if len(copies) > len(free):
            raise MemoryError(f"{len(copies)} pages are wanted and {len(free)} free")
        if copies:
            for u, j, _ in copies:
                held[u][j] = free.pop()
                users[held[u][j]] = 1
            of = dict(dtype=torch.int32, device=self.pool.device)
            pages_copy(torch.tensor([page for _, _, page in copies], **of), torch.tensor([held[u][j] for u, j, _ in copies], **of), self.pages)
        self._held, self._users, self._free = held, users, free
        at = torch.tensor(parents, device=self.pool.device)
        self.lens.copy_(self.lens.view(self.n_seqs, self.H)[at].flatten())
        if self._layers:
            self.layer_lens.copy_(self._by_layer(self._by_unit(self.layer_lens).view(self.n_seqs, self.H)[at].flatten(), n_layers))
        self._write()

    def compact(self, kept_idx, head_off, counts: Sequence[int]) -> None:
        """Thins out all sequences: unit u keeps its rows kept_idx[head_off[u] .. head_off[u + 1] - 1], counts[u] of them, as its rows 0, 1, ..
        on pages of its own, and gives the others back; lengths follow.  A unit has the rows that ``lens`` says or, with layers, ``layer_lens`` if that is more.
        There have to be pages for the rows that stay beside those that are there; with too few nothing changes."""
        import torch
        counts = [int(x) for x in counts]
        if len(counts) != len(self._held) or any(n < 0 for n in counts):
            raise ValueError("one number of rows per unit")
        need = [(n + PAGE_ROWS - 1) // PAGE_ROWS for n in counts]
        if max(need) > self.table.shape[1]:
            raise ValueError(f"a unit holds {self.table.shape[1] * PAGE_ROWS} rows")
        if sum(need) > len(self._free):
            raise MemoryError(f"{sum(need)} pages are wanted and {len(self._free)} free")
        p = self.pages
        of = (p.n_seqs, p.H, p.d, p.dtype, p.format, self.pool)
        if self._layers:                                 # (a program counts its steps in one of the two, and the other stays behind)
            p = Pages(*of, self.table, torch.maximum(self.lens, self._by_unit(self.layer_lens)))
        held = [[self._new() for _ in range(n)] for n in need]
        to = Pages(*of, self._table_of(held).to(self.pool.device), self.lens)
        try:
            pages_compact(kept_idx, head_off, sum(counts), p, to)
        except Exception:
            for pages in held:
                self._drop(pages)
            raise
        for pages in self._held:
            self._drop(pages)
        self._held = held
        self.lens.copy_(torch.tensor(counts, dtype=torch.int32))
        if self._layers:
            self.layer_lens.copy_(self._by_layer(self.lens, len(self._layers)))
        self._write()

    def _table_of(self, held):
        import torch
        host = torch.full(tuple(self.table.shape), -1, dtype=torch.int32)
        for u, h in enumerate(held):
            host[u, :len(h)] = torch.tensor(h, dtype=torch.int32)
        return host

    def _write(self) -> None:
        host = self._table_of(self._held)
        self.table.copy_(host)
        if self._layers:
            self.layer_table.copy_(self._by_layer(host, len(self._layers)))
