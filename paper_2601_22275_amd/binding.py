"""Thin ctypes binding of libvmonarch.so (argument marshalling only).

Every function takes torch CUDA tensors for device memory, hands their raw
pointers and the current HIP stream to the C ABI declared in
``include/vmonarch.h`` and ``include/vmonarch_sequence.h`` and raises ``VMonarchError`` on a non-zero return code.
No arithmetic of the method happens on the Python side, and there is no
fallback: if the shared library has not been built, importing this module's
library handle raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from ctypes import byref, c_char_p, c_float, c_int, c_size_t, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvmonarch.so")

ENTROPY_ONLINE = 0
ENTROPY_IDENTITY = 1

EXPORTS = [
    "vmonarch_version", "vmonarch_last_error", "vmonarch_set_cr_min", "vmonarch_get_cr_min",
    "vmonarch_set_entropy_mode", "vmonarch_get_entropy_mode", "vmonarch_workspace_bytes",
    "vmonarch_set_workspace", "vmonarch_shutdown", "vmonarch_attention", "vmonarch_attention_f32",
    "vmonarch_r_update", "vmonarch_r_update_f32", "vmonarch_l_update", "vmonarch_l_update_f32",
    "vmonarch_first_frame_attention", "vmonarch_first_frame_attention_f32", "vmonarch_index_maps",
    "vmonarch_permute_tokens", "vmonarch_set_phase_timing", "vmonarch_get_phase_timing",
    "vmonarch_r_update_lse", "vmonarch_r_update_lse_f32", "vmonarch_first_frame_attention_lse",
    "vmonarch_first_frame_attention_lse_f32", "vmonarch_mfma_probe", "vmonarch_entropy_attention_bwd",
    "vmonarch_entropy_attention_bwd_f32", "vmonarch_recompute_rows", "vmonarch_recompute_rows_f32",
    "vmonarch_sink_average", "vmonarch_sink_average_f32", "vmonarch_set_manual_control", "vmonarch_get_manual_control",
    "vmonarch_set_fused_apply", "vmonarch_get_fused_apply", "vmonarch_recompute_rows_noalloc",
    "vmonarch_set_flash_variant", "vmonarch_get_flash_variant",
    "vmonarch_options_init", "vmonarch_attention_ex", "vmonarch_attention_ex_f32",
    "vmonarch_recompute_tokens", "vmonarch_recompute_tokens_f32",
    "vmonarch_rotary_init", "vmonarch_rotary_scale", "vmonarch_rotary", "vmonarch_rotary_f32",
    "vmonarch_packed_attention", "vmonarch_packed_attention_f32", "vmonarch_packed_attention_bwd_workspace_bytes",
    "vmonarch_packed_attention_bwd_workspace_bytes_f32",
    "vmonarch_packed_attention_bwd", "vmonarch_packed_attention_bwd_f32", "vmonarch_paged_append", "vmonarch_paged_append_f32",
    "vmonarch_paged_attention_workspace_bytes", "vmonarch_paged_attention", "vmonarch_paged_attention_f32",
]


class VMonarchError(RuntimeError):
    pass


class Options(ctypes.Structure):
    """vmonarch_options of include/vmonarch.h: the settings and the workspace of one call."""
    _fields_ = [("struct_bytes", ctypes.c_uint32), ("cr_min", c_float), ("entropy_mode", c_int),
                ("fused_apply", c_int), ("flash_variant", c_int), ("cr_control", c_int), ("cl_control", c_int),
                ("cl_value", c_float), ("workspace", c_void_p), ("workspace_bytes", c_size_t)]


ROTARY_HALF = 0
ROTARY_INTERLEAVED = 1
ROTARY_MAX_PAIRS = 128


class Tokens(ctypes.Structure):
    """vmonarch_tokens of include/vmonarch_sequence.h: a strided token tensor."""
    _fields_ = [("data", c_void_p), ("token_stride", ctypes.c_longlong), ("head_stride", ctypes.c_longlong)]


class RotaryPlan(ctypes.Structure):
    """vmonarch_rotary_plan: which pairs of a head turn how fast."""
    _fields_ = [("struct_bytes", ctypes.c_uint32), ("layout", c_int), ("axes", c_int), ("axis_pairs", c_int * 3),
                ("amplitude", ctypes.c_double), ("frequency", ctypes.c_double * ROTARY_MAX_PAIRS)]


class Cache(ctypes.Structure):
    """vmonarch_cache: keys and values in pages, the table of pages and the lengths of the sequences."""
    _fields_ = [("k", c_void_p), ("v", c_void_p)] + [(n, ctypes.c_longlong) for n in (
        "k_page_stride", "k_token_stride", "k_head_stride", "v_page_stride", "v_token_stride", "v_head_stride")] + [
        ("n_pages", c_int), ("page_size", c_int), ("table", c_void_p), ("table_stride", ctypes.c_longlong), ("table_width", c_int),
        ("lengths", c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise VMonarchError(f"{LIB_PATH} is missing: run `python -m paper_2601_22275_amd.build` "
                                "(or __graft_entry__.build()) first")
        L = ctypes.CDLL(LIB_PATH)
        dims = [c_int] * 6
        L.vmonarch_version.restype = c_int
        L.vmonarch_last_error.restype = c_char_p
        L.vmonarch_set_cr_min.argtypes = [c_float]
        L.vmonarch_get_cr_min.restype = c_float
        L.vmonarch_set_entropy_mode.argtypes = [c_int]
        L.vmonarch_set_fused_apply.argtypes = [c_int]
        L.vmonarch_workspace_bytes.restype = c_size_t
        L.vmonarch_workspace_bytes.argtypes = dims + [c_int, c_int, c_int]
        L.vmonarch_set_workspace.argtypes = [c_void_p, c_size_t]
        L.vmonarch_set_phase_timing.argtypes = [c_int]
        L.vmonarch_get_phase_timing.argtypes = [c_void_p, c_void_p, c_void_p, c_int]
        for name in ("vmonarch_attention", "vmonarch_attention_f32"):
            getattr(L, name).argtypes = [c_void_p] * 4 + dims + [c_int, c_int, c_void_p]
        for name in ("vmonarch_r_update", "vmonarch_r_update_f32"):
            getattr(L, name).argtypes = [c_void_p] * 7 + dims + [c_float, c_float, c_void_p]
        for name in ("vmonarch_r_update_lse", "vmonarch_r_update_lse_f32"):
            getattr(L, name).argtypes = [c_void_p] * 8 + dims + [c_float, c_float, c_void_p]
        for name in ("vmonarch_first_frame_attention_lse", "vmonarch_first_frame_attention_lse_f32"):
            getattr(L, name).argtypes = [c_void_p] * 5 + dims + [c_void_p]
        for name in ("vmonarch_l_update", "vmonarch_l_update_f32"):
            getattr(L, name).argtypes = [c_void_p] * 7 + dims + [c_float, c_void_p]
        for name in ("vmonarch_first_frame_attention", "vmonarch_first_frame_attention_f32"):
            getattr(L, name).argtypes = [c_void_p] * 4 + dims + [c_void_p]
        for name in ("vmonarch_entropy_attention_bwd", "vmonarch_entropy_attention_bwd_f32"):
            getattr(L, name).argtypes = [c_void_p] * 12 + dims + [c_float, c_float, c_void_p]
        for name in ("vmonarch_recompute_tokens", "vmonarch_recompute_tokens_f32"):
            getattr(L, name).argtypes = [c_void_p] * 5 + [ctypes.c_longlong] + dims + [c_void_p]
        L.vmonarch_options_init.argtypes = [ctypes.POINTER(Options)]
        for name in ("vmonarch_attention_ex", "vmonarch_attention_ex_f32"):
            getattr(L, name).argtypes = [c_void_p] * 4 + dims + [c_int, c_int, ctypes.POINTER(Options), c_void_p]
        for name in ("vmonarch_recompute_rows", "vmonarch_recompute_rows_f32", "vmonarch_recompute_rows_noalloc"):
            getattr(L, name).argtypes = [c_void_p] * 4 + dims + [ctypes.c_longlong, ctypes.c_longlong, c_void_p]
        for name in ("vmonarch_sink_average", "vmonarch_sink_average_f32"):
            getattr(L, name).argtypes = [c_void_p] * 4 + dims + [c_void_p]
        L.vmonarch_set_manual_control.argtypes = [c_int, c_int, c_float]
        L.vmonarch_get_manual_control.argtypes = [c_void_p, c_void_p, c_void_p]
        L.vmonarch_mfma_probe.argtypes = [c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p]
        L.vmonarch_index_maps.argtypes = [c_int, c_int, c_int, c_void_p, c_void_p]
        L.vmonarch_permute_tokens.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_int,
                                              c_void_p]
        plan, n = ctypes.POINTER(RotaryPlan), ctypes.c_longlong
        L.vmonarch_rotary_init.argtypes = [plan, c_int, ctypes.c_double, c_int, c_void_p]
        L.vmonarch_rotary_scale.argtypes = [plan] + [ctypes.c_double] * 4
        for suffix in ("", "_f32"):
            getattr(L, "vmonarch_rotary" + suffix).argtypes = [c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, n, c_int, c_void_p, n, c_void_p,
                                                               c_int, c_void_p]
            getattr(L, "vmonarch_packed_attention" + suffix).argtypes = [c_void_p] * 7 + [c_int, n, n, c_int, c_int, c_int, c_float, c_int, c_void_p]
            getattr(L, "vmonarch_packed_attention_bwd" + suffix).argtypes = [c_void_p] * 11 + [c_int, n, n, c_int, c_int, c_int, c_float, c_int,
                                                                                              c_void_p, c_size_t, c_void_p]
            size = getattr(L, "vmonarch_packed_attention_bwd_workspace_bytes" + suffix)
            size.restype, size.argtypes = c_size_t, [c_int, n, n, c_int, c_int, c_int]
            getattr(L, "vmonarch_paged_append" + suffix).argtypes = [c_void_p] * 4 + [c_int, n, c_int, c_int, c_void_p, c_void_p, n, c_void_p]
            getattr(L, "vmonarch_paged_attention" + suffix).argtypes = [c_void_p] * 4 + [c_int, n, c_int, c_int, c_int, c_float, c_int, c_void_p,
                                                                                        c_size_t, c_void_p]
        L.vmonarch_paged_attention_workspace_bytes.restype = c_size_t
        L.vmonarch_paged_attention_workspace_bytes.argtypes = [c_void_p, c_int, n, c_int, c_int, c_int]
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != 0:
        raise VMonarchError(f"vmonarch error {rc}: {lib().vmonarch_last_error().decode()}")


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return c_void_p(t.data_ptr())


def _stream():
    return c_void_p(torch.cuda.current_stream().cuda_stream)


def _suffix(t: torch.Tensor) -> str:
    if t.dtype == torch.bfloat16:
        return ""
    if t.dtype == torch.float32:
        return "_f32"
    raise VMonarchError(f"unsupported dtype {t.dtype}")


def version() -> int:
    return lib().vmonarch_version()


def set_cr_min(x: float) -> None:
    _check(lib().vmonarch_set_cr_min(c_float(x)))


def get_cr_min() -> float:
    return float(lib().vmonarch_get_cr_min())


def set_manual_control(cr_control: int = 0, cl_control: int = 0, cl_value: float = float("nan")) -> None:
    _check(lib().vmonarch_set_manual_control(cr_control, cl_control, cl_value))


def get_manual_control():
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_float()
    _check(lib().vmonarch_get_manual_control(ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


def set_fused_apply(enable: bool) -> None:
    _check(lib().vmonarch_set_fused_apply(int(enable)))


def get_fused_apply() -> bool:
    return bool(lib().vmonarch_get_fused_apply())


def set_entropy_mode(mode: int) -> None:
    _check(lib().vmonarch_set_entropy_mode(mode))


def set_phase_timing(enable: bool) -> None:
    _check(lib().vmonarch_set_phase_timing(int(bool(enable))))


def get_phase_timing():
    """[(phase name, milliseconds)] of the last attention call made while timing was enabled."""
    cap = 32
    n = c_int(0)
    ms = (c_float * cap)()
    names = ctypes.create_string_buffer(cap * 32)
    _check(lib().vmonarch_get_phase_timing(ctypes.byref(n), ms, names, cap))
    return [(names.raw[32 * i:32 * i + 32].split(b"\0")[0].decode(), float(ms[i])) for i in range(n.value)]


def workspace_bytes(B, heads, T, Hs, Ws, d, iters, recompute, elem_bytes) -> int:
    return int(lib().vmonarch_workspace_bytes(B, heads, T, Hs, Ws, d, iters, int(bool(recompute)), elem_bytes))


def set_workspace(t) -> None:
    """Hand a uint8 CUDA tensor to the library as scratch (None returns to the internal arena)."""
    if t is None:
        _check(lib().vmonarch_set_workspace(None, 0))
    else:
        _check(lib().vmonarch_set_workspace(_ptr(t), t.numel() * t.element_size()))


def shutdown() -> None:
    _check(lib().vmonarch_shutdown())


def attention(q, k, v, T, Hs, Ws, iters=2, recompute=True, out=None):
    """q, k, v: [B, heads, N, d] bf16 or f32 CUDA tensors -> out of the same shape.
    recompute: False / 0 none, True / 1 first-frame recomputation, 2 sink averaging."""
    B, heads, N, d = q.shape
    assert N == T * Hs * Ws and k.shape == q.shape and v.shape == q.shape
    if out is None:
        out = torch.empty_like(q)
    fn = getattr(lib(), "vmonarch_attention" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, heads, T, Hs, Ws, d, iters, int(recompute), _stream()))
    return out


def default_options() -> Options:
    """A vmonarch_options filled with the library's defaults."""
    o = Options()
    _check(lib().vmonarch_options_init(ctypes.byref(o)))
    return o


def attention_ex(q, k, v, T, Hs, Ws, iters, recompute, options: Options, out=None, workspace=None):
    """attention() with the settings (and optionally the workspace tensor) carried by this call."""
    B, heads, N, d = q.shape
    assert N == T * Hs * Ws and k.shape == q.shape and v.shape == q.shape
    if out is None:
        out = torch.empty_like(q)
    if workspace is not None:
        options.workspace = workspace.data_ptr()
        options.workspace_bytes = workspace.numel() * workspace.element_size()
    fn = getattr(lib(), "vmonarch_attention_ex" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, heads, T, Hs, Ws, d, iters, int(recompute),
              ctypes.byref(options), _stream()))
    return out


def r_update(aR, cR, k, v, T, Hs, Ws, row_scale, cr_min):
    """Returns (aL, cL, y or None); layouts [B, heads, T*b, d] and [B, heads, T*b]."""
    B, heads, N, d = aR.shape
    aL = torch.empty_like(aR)
    cL = torch.empty((B, heads, N), dtype=torch.float32, device=aR.device)
    y = torch.empty_like(aR) if v is not None else None
    fn = getattr(lib(), "vmonarch_r_update" + _suffix(aR))
    _check(fn(_ptr(aR), _ptr(cR), _ptr(k), _ptr(v), _ptr(aL), _ptr(cL), _ptr(y), B, heads, T, Hs, Ws, d,
              c_float(row_scale), c_float(cr_min), _stream()))
    return aL, cL, y


def r_update_lse(aR, cR, k, v, T, Hs, Ws, row_scale, cr_min):
    """Like r_update; returns (aL, cL, y or None, lse) with lse [B, heads, T*b] float32."""
    B, heads, N, d = aR.shape
    aL = torch.empty_like(aR)
    cL = torch.empty((B, heads, N), dtype=torch.float32, device=aR.device)
    lse = torch.empty((B, heads, N), dtype=torch.float32, device=aR.device)
    y = torch.empty_like(aR) if v is not None else None
    fn = getattr(lib(), "vmonarch_r_update_lse" + _suffix(aR))
    _check(fn(_ptr(aR), _ptr(cR), _ptr(k), _ptr(v), _ptr(aL), _ptr(cL), _ptr(y), _ptr(lse), B, heads, T, Hs, Ws, d,
              c_float(row_scale), c_float(cr_min), _stream()))
    return aL, cL, y, lse


def l_update(q, aL, cL, y, T, Hs, Ws, q_scale):
    """Fitting sweep (y None): returns (aR, cR).  Last sweep (y given): returns out."""
    B, heads, N, d = q.shape
    fn = getattr(lib(), "vmonarch_l_update" + _suffix(q))
    if y is None:
        aR = torch.empty_like(q)
        cR = torch.empty((B, heads, N), dtype=torch.float32, device=q.device)
        _check(fn(_ptr(q), _ptr(aL), _ptr(cL), None, _ptr(aR), _ptr(cR), None, B, heads, T, Hs, Ws, d,
                  c_float(q_scale), _stream()))
        return aR, cR
    out = torch.empty_like(q)
    _check(fn(_ptr(q), _ptr(aL), _ptr(cL), _ptr(y), None, None, _ptr(out), B, heads, T, Hs, Ws, d,
              c_float(q_scale), _stream()))
    return out


def first_frame_attention(q, k, v, T, Hs, Ws, out):
    """Overwrites rows 0..b-1 of every head of `out` with exact attention over all keys."""
    B, heads, N, d = q.shape
    fn = getattr(lib(), "vmonarch_first_frame_attention" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, heads, T, Hs, Ws, d, _stream()))
    return out


def recompute_rows(q, k, v, T, Hs, Ws, out, row_begin, row_count):
    """Overwrites rows [row_begin, row_begin + row_count) of every head of `out` with exact attention over all keys."""
    B, heads, N, d = q.shape
    fn = getattr(lib(), "vmonarch_recompute_rows" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, heads, T, Hs, Ws, d, row_begin, row_count, _stream()))
    return out


def set_flash_variant(variant: int):
    _check(lib().vmonarch_set_flash_variant(int(variant)))


def get_flash_variant() -> int:
    return int(lib().vmonarch_get_flash_variant())


def recompute_tokens(q, k, v, T, Hs, Ws, out, rows):
    """Overwrites the rows listed in `rows` (int32 CUDA tensor, row numbers within a head) of every head of `out`
    with exact attention over all keys."""
    B, heads, N, d = q.shape
    assert rows.dtype == torch.int32 and rows.is_cuda and rows.is_contiguous()
    fn = getattr(lib(), "vmonarch_recompute_tokens" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(rows), rows.numel(), B, heads, T, Hs, Ws, d, _stream()))
    return out


def recompute_rows_noalloc(q, k, v, T, Hs, Ws, out, row_begin, row_count):
    """recompute_rows (bf16) through the entry point that allocates no device memory."""
    B, heads, N, d = q.shape
    assert q.dtype == torch.bfloat16
    _check(lib().vmonarch_recompute_rows_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, heads, T, Hs, Ws, d,
                                                 row_begin, row_count, _stream()))
    return out


def sink_average(q, k, v, T, Hs, Ws, out):
    """out <- (out + softmax(q K_F1^T / sqrt(d)) V_F1) / 2 in place."""
    B, heads, N, d = q.shape
    fn = getattr(lib(), "vmonarch_sink_average" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, heads, T, Hs, Ws, d, _stream()))
    return out


def first_frame_attention_lse(q, k, v, T, Hs, Ws, out):
    """Like first_frame_attention; also returns lse [B, heads, T*b] float32 (frame-0 entries written)."""
    B, heads, N, d = q.shape
    lse = torch.zeros((B, heads, N), dtype=torch.float32, device=q.device)
    fn = getattr(lib(), "vmonarch_first_frame_attention_lse" + _suffix(q))
    _check(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, heads, T, Hs, Ws, d, _stream()))
    return out, lse


def entropy_attention_bwd(q, cR, k, v, o, dO, lse, H, dH, T, Hs, Ws, row_scale, cr_min):
    """Alg. 2: returns (dq, dk, dv) for the batch of per-frame softmax blocks; dH may be None."""
    B, heads, N, d = q.shape
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    fn = getattr(lib(), "vmonarch_entropy_attention_bwd" + _suffix(q))
    _check(fn(_ptr(q), _ptr(cR), _ptr(k), _ptr(v), _ptr(o), _ptr(dO), _ptr(lse), _ptr(H), _ptr(dH), _ptr(dq), _ptr(dk),
              _ptr(dv), B, heads, T, Hs, Ws, d, c_float(row_scale), c_float(cr_min), _stream()))
    return dq, dk, dv


def mfma_probe(operands, blocks, iters):
    """Launches the matrix-instruction probe on `operands` (uint8/bf16 device tensor of blocks*512*128 bytes);
    returns (out tensor, floating-point operations of the launch)."""
    assert operands.numel() * operands.element_size() >= blocks * 512 * 128
    out = torch.empty(blocks * 512, dtype=torch.float32, device=operands.device)
    fl = ctypes.c_double(0.0)
    _check(lib().vmonarch_mfma_probe(_ptr(operands), _ptr(out), blocks, iters, ctypes.byref(fl), _stream()))
    return out, fl.value


def index_maps(T, Hs, Ws):
    """(perm, inv) as int32 CPU tensors."""
    N = T * Hs * Ws
    perm = torch.empty(N, dtype=torch.int32)
    inv = torch.empty(N, dtype=torch.int32)
    _check(lib().vmonarch_index_maps(T, Hs, Ws, c_void_p(perm.data_ptr()), c_void_p(inv.data_ptr())))
    return perm, inv


def permute_tokens(x, T, Hs, Ws, to_position_major=True, out=None):
    B, heads, N, d = x.shape
    if out is None:
        out = torch.empty_like(x)
    _check(lib().vmonarch_permute_tokens(_ptr(x), _ptr(out), B, heads, T, Hs, Ws, d * x.element_size(),
                                         int(bool(to_position_major)), _stream()))
    return out


# ---- token sequences (include/vmonarch_sequence.h) ---------------------------------------------------------------------------
#
# Token tensors are [tokens, heads, d] views with adjacent channels and any other strides.  Calls run on the tensors' device, on its
# current stream; outputs and workspaces that the caller does not bring come from torch's allocator.


def _sizes(name, x):
    """Tokens and heads of the tensor that sets the others' head size, type and device number, and those three."""
    shape = x.shape
    if len(shape) != 3:
        raise VMonarchError(f"{name}: expected [tokens, heads, d], got {tuple(shape)}")
    if not x.is_cuda:
        raise VMonarchError(f"{name}: a CUDA tensor is needed")
    n, heads, d = shape
    return n, heads, (d, x.dtype, x.get_device())


# Tokens and Cache as bytes, which ctypes passes by address: half the time of a structure and its reference
_pack_tokens = struct.Struct("@Pqq").pack
_pack_cache = struct.Struct("@PP6qiiPqiP").pack


def _tokens(name, x, like):
    """The descriptor of token tensor x, checked against like = (head size, type, device number)."""
    stride = x.stride()
    d, dtype, dev = like
    if len(stride) != 3 or x.dtype is not dtype or x.get_device() != dev or x.shape[2] != d:
        raise VMonarchError(f"{name}: expected [tokens, heads, d] of the other tensors' type, device and head size")
    if stride[2] != 1 and d > 1:
        raise VMonarchError(f"{name}: adjacent channels are needed")
    return _pack_tokens(x.data_ptr(), stride[0], stride[1])


def _int32(name, x, dev, shape):
    if x.dtype is not torch.int32 or x.get_device() != dev or x.shape != shape or not x.is_contiguous():
        raise VMonarchError(f"{name}: a contiguous int32 tensor of shape {tuple(shape)} on the other tensors' device is needed")
    return x.data_ptr()


def _same_shape(name, x, y):
    if x.shape != y.shape:
        raise VMonarchError(f"{name}: expected shape {tuple(y.shape)}, got {tuple(x.shape)}")


_entries = {}  # (name, type) -> function of the library


def _run(name, x, like, *args):
    """Calls an entry point for x's type on the current stream of its device; like = (head size, type, device number) of x."""
    _, dtype, dev = like
    fn = _entries.get((name, dtype))
    if fn is None:
        fn = _entries[name, dtype] = getattr(lib(), name + _suffix(x))
    if dev == torch.cuda.current_device():
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))  # a tenth of a microsecond; the stream object takes one
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _check(rc)


def rotary_plan(axis_pairs, base=10000.0, interleaved=False, factor=1.0, context=0.0, low_turns=0.0, high_turns=0.0, amplitude=1.0) -> RotaryPlan:
    """Rotary positions: axis_pairs[a] pairs turn with the position on axis a (one to three axes), their frequencies base^(-i / n) stretched
    for contexts `factor` times as long: all pairs alike (context = 0), or by band (see vmonarch_rotary_scale)."""
    plan = RotaryPlan()
    n = (c_int * len(axis_pairs))(*axis_pairs)
    _check(lib().vmonarch_rotary_init(ctypes.byref(plan), ROTARY_INTERLEAVED if interleaved else ROTARY_HALF, base, len(axis_pairs), n))
    if factor != 1.0:
        _check(lib().vmonarch_rotary_scale(ctypes.byref(plan), factor, context, low_turns, high_turns))
    plan.amplitude = amplitude
    return plan


def rotary(q, k, positions, plan: RotaryPlan, backward=False, q_out=None, k_out=None):
    """Turns q and k ([tokens, heads, d]; k may be None) at positions (int32 [axes, tokens], or [tokens] for one axis); backward: gradients of the
    turned tensors to those of q and k.  q_out / k_out may be q / k themselves.  Returns (q_out, k_out)."""
    n, heads, like = _sizes("q", q)
    if q_out is None:
        q_out = torch.empty_like(q)
    else:
        _same_shape("q_out", q_out, q)
    heads_k, dk, dko = 0, None, None
    if k is not None:
        if k_out is None:
            k_out = torch.empty_like(k)
        else:
            _same_shape("k_out", k_out, k)
        dk, dko, heads_k = _tokens("k", k, like), _tokens("k_out", k_out, like), k.shape[1]
        if k.shape[0] != n:
            raise VMonarchError("k: as many tokens as q are needed")
    elif k_out is not None:
        raise VMonarchError("k_out without k")
    if positions.dim() == 1:
        positions = positions[None]
    _run("vmonarch_rotary", q, like, _tokens("q", q, like), _tokens("q_out", q_out, like), heads, dk, dko, heads_k, n, like[0],
         _int32("positions", positions, like[2], (plan.axes, n)), n, byref(plan), 1 if backward else 0)
    return q_out, k_out


def packed_attention(q, k, v, q_starts, k_starts=None, causal=True, scale=None, out=None, lse=False):
    """Attention over packed sequences: q [tokens_q, heads_q, d]; k, v [tokens_k, heads_kv, d]; q_starts / k_starts int32 [n_seqs + 1] (k_starts None:
    q_starts).  scale defaults to 1 / sqrt(d).  Returns out, or (out, lse) with lse float32 [heads_q, tokens_q] for packed_attention_bwd.
    Rows of no sequence are not written: bring a cleared `out` where a padded batch's tail is read later."""
    nq, heads, like = _sizes("q", q)
    nk, kv, _ = _sizes("k", k)
    d, _, dev = like
    if out is None:
        out = q.new_empty((nq, heads, d))
    else:
        _same_shape("out", out, q)
    _same_shape("v", v, k)
    stat = torch.empty((heads, nq), dtype=torch.float32, device=q.device) if lse else None
    n = q_starts.numel()
    qs = _int32("q_starts", q_starts, dev, (n,))
    ks = qs if k_starts is None or k_starts is q_starts else _int32("k_starts", k_starts, dev, (n,))
    _run("vmonarch_packed_attention", q, like, _tokens("q", q, like), _tokens("k", k, like), _tokens("v", v, like), _tokens("out", out, like),
         stat.data_ptr() if lse else None, qs, ks, n - 1, nq, nk, heads, kv, d, 1.0 / math.sqrt(d) if scale is None else scale, 1 if causal else 0)
    return (out, stat) if lse else out


def packed_attention_bwd(q, k, v, out, d_out, lse, q_starts, k_starts=None, causal=True, scale=None, dq=None, dk=None, dv=None, workspace=None):
    """Gradients (dq, dk, dv) of packed_attention from its out and lse.  Rows of no sequence are not written (see there)."""
    nq, heads, like = _sizes("q", q)
    nk, kv, _ = _sizes("k", k)
    d, _, dev = like
    dq = q.new_empty((nq, heads, d)) if dq is None else dq
    dk = q.new_empty((nk, kv, d)) if dk is None else dk
    dv = q.new_empty((nk, kv, d)) if dv is None else dv
    if not (q.shape == out.shape == d_out.shape == dq.shape and k.shape == v.shape == dk.shape == dv.shape):
        for name, x, y in (("v", v, k), ("out", out, q), ("d_out", d_out, q), ("dq", dq, q), ("dk", dk, k), ("dv", dv, k)):
            _same_shape(name, x, y)
    if lse.dtype is not torch.float32 or lse.get_device() != dev or not lse.is_contiguous() or lse.shape != (heads, nq):
        raise VMonarchError("lse: the log-sum-exp of packed_attention is needed, float32 [heads_q, tokens_q]")
    n = q_starts.numel()
    qs = _int32("q_starts", q_starts, dev, (n,))
    ks = qs if k_starts is None or k_starts is q_starts else _int32("k_starts", k_starts, dev, (n,))
    at, size = _workspace(workspace, q, "vmonarch_packed_attention_bwd_workspace_bytes" + _suffix(q), n - 1, nq, nk, heads, kv, d)
    _run("vmonarch_packed_attention_bwd", q, like, _tokens("q", q, like), _tokens("k", k, like), _tokens("v", v, like), _tokens("out", out, like),
         _tokens("d_out", d_out, like), lse.data_ptr(), _tokens("dq", dq, like), _tokens("dk", dk, like), _tokens("dv", dv, like), qs, ks, n - 1, nq, nk,
         heads, kv, d, 1.0 / math.sqrt(d) if scale is None else scale, 1 if causal else 0, None if at is None else at.data_ptr(), size)
    return dq, dk, dv


def _workspace(given, like, name, *sizes):
    """The caller's workspace, or one of as many bytes as `name` says from torch's allocator; (tensor or None, bytes)."""
    if given is not None:
        if given.get_device() != like.get_device() or not given.is_contiguous():
            raise VMonarchError("workspace: a contiguous tensor on the other tensors' device is needed")
        return given, given.numel() * given.element_size()
    size = getattr(lib(), name)(*sizes)
    return (torch.empty(size, dtype=torch.uint8, device=like.device), size) if size else (None, 0)


def _cache(cache_k, cache_v, table, lengths, like, n_seqs):
    """The descriptor of a cache: cache_k, cache_v [pages, page_size, heads_kv, d] with adjacent channels, table int32 [n_seqs, width]."""
    d, dtype, dev = like
    shape, ks, vs = cache_k.shape, cache_k.stride(), cache_v.stride()
    if cache_v.shape != shape or len(shape) != 4 or shape[3] != d or ((ks[3] != 1 or vs[3] != 1) and d > 1):
        raise VMonarchError("cache_k, cache_v: expected [pages, page_size, heads, d] with adjacent channels, of the other tensors' head size")
    if cache_k.dtype is not dtype or cache_v.dtype is not dtype or cache_k.get_device() != dev or cache_v.get_device() != dev:
        raise VMonarchError("cache_k, cache_v: the other tensors' type and device are needed")
    width, ts = table.shape, table.stride()
    if table.dtype is not torch.int32 or table.get_device() != dev or len(width) != 2 or width[0] != n_seqs or (ts[1] != 1 and width[1] > 1):
        raise VMonarchError("table: expected int32 [n_seqs, pages of the longest] on the other tensors' device")
    return _pack_cache(cache_k.data_ptr(), cache_v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], shape[0], shape[1], table.data_ptr(), ts[0], width[1],
                       _int32("lengths", lengths, dev, (n_seqs,)))


def paged_append(k, v, cache_k, cache_v, table, q_starts, lengths, plan: RotaryPlan = None, positions=None):
    """Writes each sequence's chunk of new tokens (k, v [tokens, heads_kv, d], cut by q_starts) into the last slots of its lengths[s] tokens in the
    pages; with a plan keys are turned on the way, at `positions` or at the tokens' positions in their sequence."""
    nk, kv, like = _sizes("k", k)
    _same_shape("v", v, k)
    n = q_starts.numel()
    cache = _cache(cache_k, cache_v, table, lengths, like, n - 1)
    if cache_k.shape[2] != kv:
        raise VMonarchError("cache_k: as many heads as k are needed")
    at = None
    if positions is not None:
        if plan is None:
            raise VMonarchError("positions without a plan")
        positions = positions[None] if positions.dim() == 1 else positions
        at = _int32("positions", positions, like[2], (plan.axes, nk))
    _run("vmonarch_paged_append", k, like, _tokens("k", k, like), _tokens("v", v, like), cache, _int32("q_starts", q_starts, like[2], (n,)), n - 1, nk, kv,
         like[0],
         None if plan is None else byref(plan), at, nk)


def paged_attention(q, cache_k, cache_v, table, q_starts, lengths, causal=True, scale=None, out=None, workspace=None):
    """Attention of each sequence's chunk of new tokens (q [tokens, heads_q, d], cut by q_starts) over its lengths[s] tokens in the pages, the chunk's
    own included.  Rows of no sequence are not written (see packed_attention).  The table's width stands for the longest sequence where keys are cut into
    ranges: of one with room for far more give the columns in use, table[:, :n]."""
    nq, heads, like = _sizes("q", q)
    d, _, dev = like
    n = q_starts.numel()
    if out is None:
        out = q.new_empty((nq, heads, d))
    else:
        _same_shape("out", out, q)
    cache = _cache(cache_k, cache_v, table, lengths, like, n - 1)
    kv = cache_k.shape[2]
    at, size = _workspace(workspace, q, "vmonarch_paged_attention_workspace_bytes", cache, n - 1, nq, heads, kv, d)
    _run("vmonarch_paged_attention", q, like, _tokens("q", q, like), cache, _tokens("out", out, like), _int32("q_starts", q_starts, dev, (n,)), n - 1, nq,
         heads, kv, d, 1.0 / math.sqrt(d) if scale is None else scale, 1 if causal else 0, None if at is None else at.data_ptr(), size)
    return out
