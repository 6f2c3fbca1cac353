"""GB300 (sm_103a) block-causal attention for streaming video world models.

Python binding of the C ABI in ``include/mw_bca.h`` (argument marshalling
only; every step of the computation runs in the library's CUDA kernels).
PyTorch provides device memory and the current stream.  There is no CPU
path: without the built library every call raises.

Entry points (same names as the C ABI, taking torch tensors):
  mw_bca_fwd(q, k, v, T_chunk, scale=None, need_lse=True) -> (o, lse)
  mw_bca_bwd(q, k, v, o, lse, dout, T_chunk, scale=None) -> (dq, dk, dv)
  mw_bca_cache_fwd(q, k_new, v_new, k_cache, v_cache, cache_head, cache_len,
                   T_chunk, scale=None, need_lse=True) -> (o, lse)
  mw_bca_cache_fwd_sink(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache,
                        cache_head, cache_len, T_chunk, ...) -> (o, lse)
  mw_bca_cache_fwd_rope(..., rope_dims, rope_base, shift_frames)
  mw_bca_cache_commit(k_cache, v_cache, slot_start, k_src, v_src)
  mw_xattn_fwd(q, k, v, kv_len=None, scale=None, need_lse=True) -> (o, lse)
  mw_xattn_bwd(q, k, v, o, lse, dout, kv_len=None, scale=None) -> (dq, dk, dv)
  mw_layernorm_fwd(x, weight=None, bias=None, eps=1e-5) -> (y, mean, rstd)
  mw_layernorm_bwd(dy, x, mean, rstd, weight, bias) -> (dx, dweight, dbias)
  mw_rmsnorm_fwd(x, weight=None, residual=None, eps=1e-5) -> (y, h, rstd)
  mw_rmsnorm_quantize(x, weight=None, residual=None, eps=1e-5) -> (q, scale, h, rstd)
  mw_rmsnorm_bwd(dy, h, rstd, weight=None, dh=None) -> (dx, dweight)
  mw_quantize(x, block=(1, 128)) -> (q, scale), mw_quantize_both(x)
  mw_scaled_matmul(a, a_scale, b, b_scale, out_dtype=bf16) -> a b^T of two 8-bit forms
  mw_device_status(clear=True), mw_set_option(name, value)
Attention tensors are contiguous bf16 [B, H, rows, d] on the current CUDA device.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import math
import os
import sys
import warnings
from typing import Optional, Tuple

import torch

__all__ = [
    "MWError", "library", "lib_path", "mw_bca_fwd", "mw_bca_bwd", "mw_bca_cache_fwd",
    "mw_bca_cache_fwd_sink", "mw_bca_cache_fwd_rope", "mw_bca_cache_step",
    "mw_bca_cache_commit", "mw_bca_bwd_workspace_size", "mw_bca_bwd_head_groups",
    "mw_bca_cache_workspace_size",
    "mw_device_status", "mw_set_option", "mw_qkv_rope_split", "BlockCausalAttention",
    "mw_xattn_fwd", "mw_xattn_bwd", "mw_xattn_workspace_size", "mw_xattn_bwd_workspace_size",
    "mw_layernorm_fwd", "mw_layernorm_bwd", "mw_layernorm_bwd_workspace_size", "CrossAttention",
    "LayerNorm", "mw_rmsnorm_fwd", "mw_rmsnorm_quantize", "mw_rmsnorm_bwd",
    "mw_rmsnorm_bwd_workspace_size", "mw_quantize", "mw_quantize_both", "mw_scaled_matmul",
    "RMSNorm", "Fp8Linear",
    "EXPORTED_SYMBOLS",
    "RingState",
]

_PKG = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_PKG, "_lib", "libmw_bca.so")
_native_path = os.path.join(_PKG, "_lib", "_mw_torch.so")

EXPORTED_SYMBOLS = (
    "mw_bca_fwd", "mw_bca_bwd_workspace_size", "mw_bca_bwd", "mw_bca_bwd_stage",
    "mw_bca_cache_workspace_size",
    "mw_bca_cache_fwd", "mw_bca_cache_commit", "mw_status_string", "mw_last_error",
    "mw_device_status", "mw_set_option", "mw_bca_cache_fwd_noalloc", "mw_bca_cache_fwd_sink",
    "mw_bca_cache_fwd_rope", "mw_qkv_rope_split", "mw_bca_cache_step", "mw_bca_bwd_head_groups",
    "mw_xattn_workspace_size", "mw_xattn_fwd", "mw_xattn_bwd_workspace_size", "mw_xattn_bwd",
    "mw_layernorm_fwd", "mw_layernorm_bwd_workspace_size", "mw_layernorm_bwd",
    "mw_rmsnorm_fwd", "mw_rmsnorm_bwd_workspace_size", "mw_rmsnorm_bwd", "mw_quantize",
    "mw_scaled_matmul",
)

STATUS = {0: "MW_OK", 1: "MW_ERR_INVALID_ARG", 2: "MW_ERR_UNSUPPORTED", 3: "MW_ERR_CUDA",
          4: "MW_ERR_TIMEOUT", 5: "MW_ERR_WORKSPACE"}


class MWError(RuntimeError):
    """A non-zero mw_status from the library, with mw_last_error()'s text."""

    def __init__(self, code: int, message: str):
        super().__init__(f"{STATUS.get(code, code)}: {message}")
        self.code = code


_lib: Optional[ctypes.CDLL] = None
# csrc/mw_torch.cpp: the common forms of the calls below with their checks and
# allocations in native code.  Calls that the host bounds, a call's wall time:
# forward of 2 heads x 256 tokens 20.6 -> 6.8 us, streaming step against one
# committed chunk 43.0 -> 15.9 us, forward and backward of 16 heads x 1760
# tokens through autograd 286 -> 173 us.  Each function returns None for
# arguments it does not take; the checks here then follow.  None until the
# library is loaded, or when the module was not built.
_native = None

_P = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float
_Z = ctypes.c_size_t
_L = ctypes.c_longlong


def library() -> ctypes.CDLL:
    """The loaded C library (raises when it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(lib_path):
        raise RuntimeError(
            f"{lib_path} is missing: build it with `python -c 'import __graft_entry__ as g; "
            "g.build()'` (there is no CPU fallback)")
    lib = ctypes.CDLL(lib_path)
    sig = {
        "mw_bca_fwd": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_bwd_workspace_size": (_Z, [_I, _I, _I, _I, _I]),
        "mw_bca_bwd_head_groups": (_I, [_I, _I, _I, _I, _I, _I]),
        "mw_bca_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _Z,
                            _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_bwd_stage": (_I, [_I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _Z,
                                  _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_cache_workspace_size": (_Z, [_I, _I, _I, _I, _I, _I]),
        "mw_bca_cache_fwd": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _Z,
                                  _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_cache_fwd_sink": (_I, [_P, _P, _P, _P, _P, _I, _P, _P, _I, _I, _I, _P, _P, _P,
                                       _Z, _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_cache_fwd_rope": (_I, [_P, _P, _P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _F, _I,
                                       _P, _P, _P, _Z, _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_cache_commit": (_I, [_P, _P, _I, _I, _P, _P, _I, _I, _I, _I, _P]),
        "mw_qkv_rope_split": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _I, _I, _P]),
        "mw_bca_cache_step": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _Z,
                                   _I, _I, _I, _I, _I, _F, _P]),
        "mw_bca_cache_fwd_noalloc": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _P, _P,
                                          _I, _I, _I, _I, _I, _F, _P]),
        "mw_xattn_workspace_size": (_Z, [_I, _I, _I, _I, _I, _I]),
        "mw_xattn_fwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _Z, _I, _I, _I, _I, _I, _I, _F, _P]),
        "mw_xattn_bwd_workspace_size": (_Z, [_I, _I, _I, _I, _I, _I]),
        "mw_xattn_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _Z,
                              _I, _I, _I, _I, _I, _I, _F, _P]),
        "mw_layernorm_fwd": (_I, [_P, _P, _P, _P, _P, _P, _L, _I, _I, _F, _I, _I, _I, _P]),
        "mw_layernorm_bwd_workspace_size": (_Z, [_L, _I, _I]),
        "mw_layernorm_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _Z, _L, _I, _I,
                                  _I, _I, _I, _P]),
        "mw_rmsnorm_fwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _L, _I, _I, _F, _I, _I, _I, _P]),
        "mw_rmsnorm_bwd_workspace_size": (_Z, [_L, _I, _I]),
        "mw_rmsnorm_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _Z, _L, _I, _I, _I, _I, _I, _P]),
        "mw_quantize": (_I, [_P, _P, _P, _P, _P, _L, _I, _I, _I, _P]),
        "mw_scaled_matmul": (_I, [_P, _P, _I, _I, _P, _P, _I, _I, _P, _I, _I, _I, _I, _P]),
        "mw_status_string": (ctypes.c_char_p, [_I]),
        "mw_last_error": (ctypes.c_char_p, []),
        "mw_device_status": (_I, [_P, _I]),
        "mw_set_option": (_I, [ctypes.c_char_p, ctypes.c_longlong]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    _load_native(lib)
    return lib


def _load_native(lib: ctypes.CDLL) -> None:
    global _native

    def without(why: str) -> None:
        warnings.warn(f"{_native_path} {why}: calls go the longer way, two to three times as long "
                      "for small ones; build again", RuntimeWarning, stacklevel=4)

    if not os.path.exists(_native_path):
        return without("is missing")
    loader = importlib.machinery.ExtensionFileLoader("_mw_torch", _native_path)
    try:
        module = importlib.util.module_from_spec(
            importlib.util.spec_from_loader("_mw_torch", loader))
        loader.exec_module(module)
    except ImportError as e:
        return without(f"was not loaded ({e})")
    # it reads PyTorch's objects through the headers it was built with
    built = getattr(module, "torch_version", None), getattr(module, "python_hexversion", 0)
    running = str(torch.__version__), sys.hexversion
    if built != running:
        return without(f"was built for PyTorch {built[0]} and Python {built[1]:#x}, not PyTorch "
                       f"{running[0]} and Python {running[1]:#x}")
    module.bind(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in (
        "mw_bca_fwd", "mw_bca_bwd", "mw_bca_bwd_workspace_size", "mw_bca_cache_workspace_size",
        "mw_bca_cache_fwd_rope", "mw_bca_cache_step", "mw_qkv_rope_split",
        "mw_xattn_workspace_size", "mw_xattn_fwd", "mw_xattn_bwd_workspace_size", "mw_xattn_bwd",
        "mw_layernorm_fwd", "mw_layernorm_bwd_workspace_size", "mw_layernorm_bwd",
        "mw_rmsnorm_fwd", "mw_rmsnorm_bwd_workspace_size", "mw_rmsnorm_bwd", "mw_quantize",
        "mw_scaled_matmul", "mw_last_error")), MWError)
    _native = module


def _check(code: int) -> None:
    if code != 0:
        msg = library().mw_last_error().decode(errors="replace")
        raise MWError(code, msg)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _bhnd(t: torch.Tensor, name: str) -> Tuple[int, int, int, int]:
    """Shape of a contiguous bf16 [B, H, rows, d] tensor (its device is
    checked by _on_device, once every shape is known to be right)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be bfloat16, got {t.dtype}")
    if t.dim() != 4 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [B, H, rows, d] tensor")
    return tuple(t.shape)  # type: ignore[return-value]


def _expect(t, name: str, shape, dtype=torch.bfloat16) -> None:
    """A caller-supplied output buffer: exactly this shape and dtype,
    contiguous.  The library cannot see buffer sizes, so a short buffer
    would be written past its end."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_contiguous() \
            or tuple(t.shape) != tuple(shape):
        got = (f"{t.dtype} {tuple(t.shape)}" + ("" if t.is_contiguous() else " non-contiguous")
               if isinstance(t, torch.Tensor) else type(t).__name__)
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, "
                         f"got {got}")


def _chunks(rows: int, T_chunk: int, what: str) -> int:
    if int(T_chunk) < 1:
        raise ValueError(f"T_chunk must be >= 1, got {T_chunk}")
    if rows % T_chunk != 0:
        raise ValueError(f"{what} {rows} is not a multiple of T_chunk={T_chunk}")
    return rows // T_chunk


def _on_device(ref: torch.Tensor, named) -> None:
    """Every tensor on ref's CUDA device, and that device current (the
    library launches on the current device and stream)."""
    if not ref.is_cuda:
        raise ValueError("the tensors must be CUDA tensors (there is no CPU path)")
    for name, t in named:
        if t is not None and t.device != ref.device:
            raise ValueError(f"{name} is on {t.device}, the other tensors on {ref.device}")
    if ref.device.index != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {ref.device} but the current device is "
                         f"cuda:{torch.cuda.current_device()}: call under torch.cuda.device")


def _no_alias(outputs, inputs) -> None:
    """No output buffer shares bytes with an input or with another output
    (the kernels read inputs while they write outputs)."""
    spans = []
    for kind, group in (("output", outputs), ("input", inputs)):
        for name, t in group:
            if t is not None and t.numel() > 0:
                p = t.data_ptr()
                spans.append((f"{kind} {name}", p, p + t.numel() * t.element_size()))
    n_out = sum(1 for _, t in outputs if t is not None and t.numel() > 0)
    for a in range(n_out):
        for b in range(a + 1, len(spans)):
            if spans[a][1] < spans[b][2] and spans[b][1] < spans[a][2]:
                raise ValueError(f"{spans[a][0]} overlaps {spans[b][0]}")


def _workspace(ws: Optional[torch.Tensor], nbytes: int,
               device: torch.device) -> Optional[torch.Tensor]:
    """At least nbytes of device scratch (None when none is needed): the
    caller's buffer when it is large enough, else a new one."""
    if nbytes == 0:
        return None
    if ws is not None:
        if not ws.is_contiguous():
            raise ValueError("workspace must be contiguous")
        if ws.numel() * ws.element_size() >= nbytes:
            return ws
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _scale(scale: Optional[float], d: int) -> float:
    return 1.0 / math.sqrt(d) if scale is None else float(scale)


def mw_bca_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, T_chunk: int,
               scale: Optional[float] = None, need_lse: bool = True,
               out: Optional[Tuple[torch.Tensor, Optional[torch.Tensor]]] = None
               ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Block-causal attention forward (Sec. 3.2); returns (O, LSE or None).

    ``out`` = (o, lse) reuses caller buffers (lse may be None)."""
    if out is None and _native is not None:
        r = _native.fwd(q, k, v, T_chunk, scale, need_lse)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    B, H, N, d = _bhnd(q, "q")
    for t, n in ((k, "k"), (v, "v")):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape {tuple(t.shape)} != q shape {(B, H, N, d)}")
    n_chunks = _chunks(N, T_chunk, "sequence length")
    o, lse = out if out is not None else (None, None)
    if out is not None:
        _expect(o, "o", (B, H, N, d))
        if lse is not None:
            _expect(lse, "lse", (B, H, N), torch.float32)
    _on_device(q, (("k", k), ("v", v), ("o", o), ("lse", lse)))
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device) if need_lse else None
    else:
        _no_alias((("o", o), ("lse", lse)), (("q", q), ("k", k), ("v", v)))
    _check(library().mw_bca_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H,
                                n_chunks, T_chunk, d, _scale(scale, d), _stream()))
    return o, lse


def mw_bca_bwd_workspace_size(B: int, H: int, n_chunks: int, T_chunk: int, d: int) -> int:
    return int(library().mw_bca_bwd_workspace_size(B, H, n_chunks, T_chunk, d))


def mw_bca_bwd_head_groups(B: int, H: int, n_chunks: int, T_chunk: int, d: int,
                           sm_count: int = 0) -> int:
    """Head groups of the backward's CTA order for these sizes (B*H = head by
    head); host-side planning only."""
    g = int(library().mw_bca_bwd_head_groups(B, H, n_chunks, T_chunk, d, sm_count))
    if g < 0:
        raise MWError(1, library().mw_last_error().decode(errors="replace"))
    return g


def mw_bca_bwd(q, k, v, o, lse, dout, T_chunk: int, scale: Optional[float] = None,
               workspace: Optional[torch.Tensor] = None, stage: int = 0, out=None):
    """Gradients (dQ, dK, dV) of sum(O * dout) through mw_bca_fwd.

    ``stage`` 1/2/3 runs one stage of the backward (see mw_bca_bwd_stage);
    ``out`` = (dq, dk, dv) preallocated outputs."""
    if out is None and workspace is None and stage == 0 and _native is not None:
        r = _native.bwd(q, k, v, o, lse, dout, T_chunk, scale)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    B, H, N, d = _bhnd(q, "q")
    for t, n in ((k, "k"), (v, "v"), (o, "o"), (dout, "dout")):
        if _bhnd(t, n) != (B, H, N, d):
            raise ValueError(f"{n} shape {tuple(t.shape)} != q shape {(B, H, N, d)}")
    _expect(lse, "lse", (B, H, N), torch.float32)
    n = _chunks(N, T_chunk, "sequence length")
    dq, dk, dv = out if out is not None else (None, None, None)
    if out is not None:
        for t, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
            _expect(t, name, (B, H, N, d))
    _on_device(q, (("k", k), ("v", v), ("o", o), ("lse", lse), ("dout", dout), ("dq", dq),
                   ("dk", dk), ("dv", dv), ("workspace", workspace)))
    ws_bytes = mw_bca_bwd_workspace_size(B, H, n, T_chunk, d)
    workspace = _workspace(workspace, ws_bytes, q.device)
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    _no_alias((("dq", dq), ("dk", dk), ("dv", dv), ("workspace", workspace)),
              (("q", q), ("k", k), ("v", v), ("o", o), ("lse", lse), ("dout", dout)))
    _check(library().mw_bca_bwd_stage(stage, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                      _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                      ws_bytes, B, H, n, T_chunk, d, _scale(scale, d), _stream()))
    return dq, dk, dv


def mw_bca_cache_workspace_size(B: int, H: int, n_q_chunks: int, T_chunk: int, d: int,
                                cache_len: int) -> int:
    return int(library().mw_bca_cache_workspace_size(B, H, n_q_chunks, T_chunk, d, cache_len))


def mw_bca_cache_fwd(q, k_new, v_new, k_cache, v_cache, cache_head: int, cache_len: int,
                     T_chunk: int, scale: Optional[float] = None, need_lse: bool = True,
                     workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """In-flight chunks against the rolling KV cache (Sec. 3.5); returns (O, LSE or None)."""
    return _cache_fwd(q, k_new, v_new, None, None, k_cache, v_cache, cache_head, cache_len,
                      T_chunk, scale, need_lse, workspace, out)


def mw_bca_cache_fwd_sink(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, cache_head: int,
                          cache_len: int, T_chunk: int, scale: Optional[float] = None,
                          need_lse: bool = True, workspace: Optional[torch.Tensor] = None,
                          out: Optional[torch.Tensor] = None):
    """As mw_bca_cache_fwd with a sink anchor k_sink / v_sink [B, H, S, d] that
    every in-flight chunk sees ahead of the ring (Sec. 3.5); returns (O, LSE or None)."""
    return _cache_fwd(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, cache_head, cache_len,
                      T_chunk, scale, need_lse, workspace, out)


def mw_bca_cache_fwd_rope(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, cache_head: int,
                          cache_len: int, T_chunk: int, rope_dims: int, rope_base: float,
                          shift_frames: int, scale: Optional[float] = None,
                          need_lse: bool = True, workspace: Optional[torch.Tensor] = None,
                          out: Optional[torch.Tensor] = None):
    """As mw_bca_cache_fwd_sink (k_sink may be None) with RoPE re-shifting
    (Sec. 3.5): queries, in-flight and ring keys rotated at their stream
    positions, the sink at its own, ``shift_frames`` frames evicted; the
    sink's keys turn forward by the shift as they are read.  Returns
    (O, LSE or None)."""
    return _cache_fwd(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, cache_head, cache_len,
                      T_chunk, scale, need_lse, workspace, out,
                      rope=(rope_dims, rope_base, shift_frames))


def _cache_fwd(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, cache_head, cache_len,
               T_chunk, scale, need_lse, workspace, out, rope=None, commit=None):
    if out is None and _native is not None:
        r = _native.cache(q, k_new, v_new, k_sink, v_sink, k_cache, v_cache, cache_head, cache_len,
                          T_chunk, scale, need_lse, workspace, rope, commit)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    B, H, M, d = _bhnd(q, "q")
    for t, n in ((k_new, "k_new"), (v_new, "v_new")):
        if _bhnd(t, n) != (B, H, M, d):
            raise ValueError(f"{n} shape {tuple(t.shape)} != q shape {(B, H, M, d)}")
    Bc, Hc, cap, dc = _bhnd(k_cache, "k_cache")
    if (Bc, Hc, dc) != (B, H, d) or tuple(v_cache.shape) != tuple(k_cache.shape):
        raise ValueError("k_cache / v_cache must be [B, H, cap, d] matching q")
    _bhnd(v_cache, "v_cache")
    W = _chunks(M, T_chunk, "query rows")
    sink_len = 0
    if k_sink is not None:
        Bs, Hs, sink_len, ds = _bhnd(k_sink, "k_sink")
        _bhnd(v_sink, "v_sink")
        if (Bs, Hs, ds) != (B, H, d) or tuple(v_sink.shape) != tuple(k_sink.shape):
            raise ValueError("k_sink / v_sink must be [B, H, S, d] matching q")
    if out is not None:
        _expect(out, "out", (B, H, M, d))
    _on_device(q, (("k_new", k_new), ("v_new", v_new), ("k_cache", k_cache),
                   ("v_cache", v_cache), ("k_sink", k_sink), ("v_sink", v_sink), ("out", out),
                   ("workspace", workspace)))
    ws_bytes = mw_bca_cache_workspace_size(B, H, W, T_chunk, d, sink_len + cache_len)
    workspace = _workspace(workspace, ws_bytes, q.device)
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((B, H, M), dtype=torch.float32, device=q.device) if need_lse else None
    # the streaming step also writes the ring (its commit)
    ring = (("k_cache", k_cache), ("v_cache", v_cache))
    _no_alias((("out", o), ("lse", lse), ("workspace", workspace))
              + (ring if commit is not None else ()),
              (("q", q), ("k_new", k_new), ("v_new", v_new), ("k_sink", k_sink),
               ("v_sink", v_sink)) + (ring if commit is None else ()))
    if commit is not None:
        _check(library().mw_bca_cache_step(
            _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), cap, cache_head,
            cache_len, int(commit[0]), int(commit[1]), _ptr(o), _ptr(lse),
            _ptr(workspace), ws_bytes, B, H, W, T_chunk, d,
            _scale(scale, d), _stream()))
    elif rope is not None:
        _check(library().mw_bca_cache_fwd_rope(
            _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_sink), _ptr(v_sink), sink_len,
            _ptr(k_cache), _ptr(v_cache), cap, cache_head, cache_len, int(rope[0]),
            float(rope[1]), int(rope[2]), _ptr(o), _ptr(lse),
            _ptr(workspace), ws_bytes, B, H, W, T_chunk, d,
            _scale(scale, d), _stream()))
    elif k_sink is None:
        _check(library().mw_bca_cache_fwd(
            _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), cap, cache_head,
            cache_len, _ptr(o), _ptr(lse), _ptr(workspace), ws_bytes,
            B, H, W, T_chunk, d, _scale(scale, d), _stream()))
    else:
        _check(library().mw_bca_cache_fwd_sink(
            _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_sink), _ptr(v_sink), sink_len,
            _ptr(k_cache), _ptr(v_cache), cap, cache_head, cache_len, _ptr(o), _ptr(lse),
            _ptr(workspace), ws_bytes, B, H, W, T_chunk, d,
            _scale(scale, d), _stream()))
    return o, lse


def mw_bca_cache_step(q, k_new, v_new, k_cache, v_cache, cache_head: int, cache_len: int,
                      commit_slot: int, commit_rows: int, T_chunk: int,
                      scale: Optional[float] = None, need_lse: bool = True,
                      workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """One streaming step (Sec. 3.5): mw_bca_cache_fwd, then the first
    ``commit_rows`` rows of k_new / v_new go to ring rows (commit_slot + r) mod
    cap (FIFO eviction); returns (O, LSE or None)."""
    return _cache_fwd(q, k_new, v_new, None, None, k_cache, v_cache, cache_head, cache_len,
                      T_chunk, scale, need_lse, workspace, out,
                      commit=(commit_slot, commit_rows))


def mw_bca_cache_commit(k_cache, v_cache, slot_start: int, k_src, v_src) -> None:
    """Write k_src / v_src rows at ring rows (slot_start + r) mod cap (Sec. 3.5)."""
    B, H, cap, d = _bhnd(k_cache, "k_cache")
    _bhnd(v_cache, "v_cache")
    Bs, Hs, rows, ds = _bhnd(k_src, "k_src")
    _bhnd(v_src, "v_src")
    if (Bs, Hs, ds) != (B, H, d) or tuple(v_src.shape) != tuple(k_src.shape):
        raise ValueError("k_src / v_src must be [B, H, rows, d] matching the cache")
    if tuple(v_cache.shape) != (B, H, cap, d):
        raise ValueError("k_cache / v_cache must have the same shape")
    _on_device(k_cache, (("v_cache", v_cache), ("k_src", k_src), ("v_src", v_src)))
    _no_alias((("k_cache", k_cache), ("v_cache", v_cache)), (("k_src", k_src), ("v_src", v_src)))
    _check(library().mw_bca_cache_commit(_ptr(k_cache), _ptr(v_cache), cap, slot_start,
                                         _ptr(k_src), _ptr(v_src), rows, B, H, d, _stream()))


def mw_qkv_rope_split(qkv: torch.Tensor, rope_dims: int = 0, rope_base: float = 10000.0,
                      tokens_per_frame: int = 1, first_frame: int = 0,
                      out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None
                      ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Split a fused QKV projection [B, N, 3, H, d] into head-major Q, K, V
    [B, H, N, d], turning the first ``rope_dims`` channels of Q and K by their
    frame's temporal rotary angle (token t at frame first_frame + t //
    tokens_per_frame; Sec. 3.2 inputs, Sec. 3.5 positions)."""
    if out is None and _native is not None:
        r = _native.qkv(qkv, rope_dims, rope_base, tokens_per_frame, first_frame)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    if not isinstance(qkv, torch.Tensor) or qkv.dtype != torch.bfloat16:
        raise TypeError("qkv must be a bfloat16 tensor")
    if qkv.dim() != 5 or qkv.shape[2] != 3 or not qkv.is_contiguous():
        raise ValueError("qkv must be a contiguous [B, N, 3, H, d] tensor")
    B, N, _, H, d = qkv.shape
    if out is not None:
        if len(out) != 3:
            raise ValueError("out must be (q, k, v)")
        for t, name in zip(out, ("q", "k", "v")):
            _expect(t, name, (B, H, N, d))
    _on_device(qkv, tuple(zip(("q", "k", "v"), out)) if out is not None else ())
    if out is None:
        out = tuple(torch.empty(B, H, N, d, dtype=torch.bfloat16, device=qkv.device)
                    for _ in range(3))
    q, k, v = out
    _no_alias((("q", q), ("k", k), ("v", v)), (("qkv", qkv),))
    _check(library().mw_qkv_rope_split(_ptr(qkv), _ptr(q), _ptr(k), _ptr(v), B, N, H, d,
                                       int(rope_dims), float(rope_base), int(tokens_per_frame),
                                       int(first_frame), _stream()))
    return q, k, v


def _xattn_shapes(q, k, v, kv_len):
    """B, H, Hkv, M, S, d of a cross attention call."""
    B, H, M, d = _bhnd(q, "q")
    Bk, Hkv, S, dk = _bhnd(k, "k")
    if _bhnd(v, "v") != (Bk, Hkv, S, dk):
        raise ValueError(f"v shape {tuple(v.shape)} != k shape {tuple(k.shape)}")
    if (Bk, dk) != (B, d):
        raise ValueError(f"k shape {tuple(k.shape)} does not match q shape {tuple(q.shape)}")
    if Hkv < 1 or H % Hkv != 0:
        raise ValueError(f"q has {H} heads, not a multiple of k's {Hkv}")
    if kv_len is not None:
        _expect(kv_len, "kv_len", (B,), torch.int32)
    return B, H, Hkv, M, S, d


def mw_xattn_workspace_size(B: int, H: int, Hkv: int, M: int, S: int, d: int) -> int:
    return int(library().mw_xattn_workspace_size(B, H, Hkv, M, S, d))


def mw_xattn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                 kv_len: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                 need_lse: bool = True, workspace: Optional[torch.Tensor] = None,
                 out: Optional[Tuple[torch.Tensor, Optional[torch.Tensor]]] = None
                 ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Cross attention of q [B, H, M, d] to an encoder's states k, v
    [B, Hkv, S, d]: H / Hkv query heads share a head of K and V, and of a sample's
    states the first ``kv_len`` [B] (int32, on the device) count; returns (O, LSE
    or None), O = 0 and LSE = -inf for a sample without states.

    ``out`` = (o, lse) reuses caller buffers (lse may be None)."""
    if out is None and _native is not None:
        r = _native.xattn_fwd(q, k, v, kv_len, scale, need_lse, workspace)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    B, H, Hkv, M, S, d = _xattn_shapes(q, k, v, kv_len)
    o, lse = out if out is not None else (None, None)
    if out is not None:
        _expect(o, "o", (B, H, M, d))
        if lse is not None:
            _expect(lse, "lse", (B, H, M), torch.float32)
    _on_device(q, (("k", k), ("v", v), ("kv_len", kv_len), ("o", o), ("lse", lse),
                   ("workspace", workspace)))
    ws_bytes = mw_xattn_workspace_size(B, H, Hkv, M, S, d)
    workspace = _workspace(workspace, ws_bytes, q.device)
    if out is None:
        o = torch.empty_like(q)
        lse = torch.empty((B, H, M), dtype=torch.float32, device=q.device) if need_lse else None
    _no_alias((("o", o), ("lse", lse), ("workspace", workspace)),
              (("q", q), ("k", k), ("v", v), ("kv_len", kv_len)))
    _check(library().mw_xattn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(kv_len), _ptr(o), _ptr(lse),
                                  _ptr(workspace), ws_bytes, B, H, Hkv, M, S, d,
                                  _scale(scale, d), _stream()))
    return o, lse


def mw_xattn_bwd_workspace_size(B: int, H: int, Hkv: int, M: int, S: int, d: int) -> int:
    return int(library().mw_xattn_bwd_workspace_size(B, H, Hkv, M, S, d))


def mw_xattn_bwd(q, k, v, o, lse, dout, kv_len: Optional[torch.Tensor] = None,
                 scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None, out=None):
    """Gradients (dQ, dK, dV) of sum(O * dout) through mw_xattn_fwd; those of K and
    V are sums over the query heads that share them, and 0 past ``kv_len``.

    ``out`` = (dq, dk, dv) preallocated outputs."""
    if out is None and workspace is None and _native is not None:
        r = _native.xattn_bwd(q, k, v, o, lse, dout, kv_len, scale)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    B, H, Hkv, M, S, d = _xattn_shapes(q, k, v, kv_len)
    for t, n in ((o, "o"), (dout, "dout")):
        if _bhnd(t, n) != (B, H, M, d):
            raise ValueError(f"{n} shape {tuple(t.shape)} != q shape {(B, H, M, d)}")
    _expect(lse, "lse", (B, H, M), torch.float32)
    dq, dk, dv = out if out is not None else (None, None, None)
    if out is not None:
        _expect(dq, "dq", (B, H, M, d))
        _expect(dk, "dk", (B, Hkv, S, d))
        _expect(dv, "dv", (B, Hkv, S, d))
    _on_device(q, (("k", k), ("v", v), ("kv_len", kv_len), ("o", o), ("lse", lse), ("dout", dout),
                   ("dq", dq), ("dk", dk), ("dv", dv), ("workspace", workspace)))
    ws_bytes = mw_xattn_bwd_workspace_size(B, H, Hkv, M, S, d)
    workspace = _workspace(workspace, ws_bytes, q.device)
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    _no_alias((("dq", dq), ("dk", dk), ("dv", dv), ("workspace", workspace)),
              (("q", q), ("k", k), ("v", v), ("o", o), ("lse", lse), ("dout", dout),
               ("kv_len", kv_len)))
    _check(library().mw_xattn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(kv_len), _ptr(o), _ptr(lse),
                                  _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                  ws_bytes, B, H, Hkv, M, S, d, _scale(scale, d), _stream()))
    return dq, dk, dv


_NORM_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def _norm_type(t, name: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in _NORM_TYPES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    return _NORM_TYPES[t.dtype]


def _norm_params(x, weight, bias):
    """Rows, channels, groups and the parameters' type of a layer norm call."""
    if x.dim() < 1 or not x.is_contiguous():
        raise ValueError("x must be a contiguous [..., C] tensor")
    C = x.shape[-1]
    rows = x.numel() // C if C else 0
    groups, ptype, shape = 1, 1, None
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        kind = _norm_type(t, name)
        if t.dim() not in (1, 2) or t.shape[-1] != C or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous [C] or [groups, C] tensor, C = {C}, "
                             f"got {tuple(t.shape)}")
        if shape is not None and (tuple(t.shape) != shape or kind != ptype):
            raise ValueError("weight and bias must have one shape and type")
        shape, ptype = tuple(t.shape), kind
        groups = t.shape[0] if t.dim() == 2 else 1
    if groups < 1 or rows % groups:
        raise ValueError(f"{rows} rows are not a multiple of the {groups} groups of weight or bias")
    return rows, C, groups, ptype


def mw_layernorm_fwd(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
                     bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                     out_dtype: Optional[torch.dtype] = None, need_stats: bool = True,
                     out: Optional[torch.Tensor] = None):
    """Layer norm over the last dimension of x [..., C] (bf16 or fp32); returns
    (y, mean, rstd), the latter two fp32 [...] or None.

    ``weight`` and ``bias``: [C], or [groups, C] with one of each for every one of
    ``groups`` equal runs of consecutive rows (samples, frames), or None.  y has
    ``out_dtype`` (None: x's; fp32 only with x in fp32)."""
    if out is None and _native is not None:
        r = _native.norm_fwd(x, weight, bias, eps, out_dtype, need_stats)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt = _norm_type(x, "x")
    rows, C, groups, ptype = _norm_params(x, weight, bias)
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in _NORM_TYPES:
        raise TypeError(f"out_dtype must be bfloat16 or float32, got {out_dtype}")
    if out is not None:
        _expect(out, "out", tuple(x.shape), out_dtype)
    _on_device(x, (("weight", weight), ("bias", bias), ("out", out)))
    y = torch.empty(x.shape, dtype=out_dtype, device=x.device) if out is None else out
    mean = rstd = None
    if need_stats:
        mean, rstd = (torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
                      for _ in range(2))
    _no_alias((("out", y),), (("x", x), ("weight", weight), ("bias", bias)))
    _check(library().mw_layernorm_fwd(_ptr(x), _ptr(weight), _ptr(bias), _ptr(y), _ptr(mean),
                                      _ptr(rstd), rows, C, groups, float(eps), xt,
                                      _NORM_TYPES[out_dtype], ptype, _stream()))
    return y, mean, rstd


def mw_layernorm_bwd_workspace_size(rows: int, C: int, groups: int) -> int:
    return int(library().mw_layernorm_bwd_workspace_size(rows, C, groups))


def mw_layernorm_bwd(dy, x, mean, rstd, weight: Optional[torch.Tensor] = None,
                     bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients (dx, dweight, dbias) of sum(y * dy) through mw_layernorm_fwd, None
    in the place of a parameter that is None (bias: only its shape is used)."""
    if workspace is None and _native is not None:
        r = _native.norm_bwd(dy, x, mean, rstd, weight, bias)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt, yt = _norm_type(x, "x"), _norm_type(dy, "dy")
    rows, C, groups, ptype = _norm_params(x, weight, bias)
    _expect(dy, "dy", tuple(x.shape), dy.dtype)
    for t, name in ((mean, "mean"), (rstd, "rstd")):
        _expect(t, name, tuple(x.shape[:-1]), torch.float32)
    _on_device(x, (("dy", dy), ("mean", mean), ("rstd", rstd), ("weight", weight), ("bias", bias),
                   ("workspace", workspace)))
    params = weight is not None or bias is not None
    ws_bytes = mw_layernorm_bwd_workspace_size(rows, C, groups) if params else 0
    workspace = _workspace(workspace, ws_bytes, x.device)
    dx = torch.empty_like(x)
    dw = None if weight is None else torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    _no_alias((("workspace", workspace),), (("dy", dy), ("x", x), ("mean", mean), ("rstd", rstd),
                                            ("weight", weight)))
    _check(library().mw_layernorm_bwd(_ptr(dy), _ptr(x), _ptr(mean), _ptr(rstd), _ptr(weight),
                                      _ptr(dx), _ptr(dw), _ptr(db), _ptr(workspace), ws_bytes,
                                      rows, C, groups, xt, yt, ptype, _stream()))
    return dx, dw, db


_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _rms_inputs(x, weight, residual):
    xt = _norm_type(x, "x")
    rows, C, groups, ptype = _norm_params(x, weight, None)
    if residual is not None:
        _expect(residual, "residual", tuple(x.shape), x.dtype)
    return xt, rows, C, groups, ptype


def mw_rmsnorm_fwd(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
                   residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                   out_dtype: Optional[torch.dtype] = None, need_stats: bool = True,
                   out: Optional[torch.Tensor] = None):
    """Root-mean-square norm over the last dimension of h = x + residual (bf16 or fp32, the
    sum rounded to x's type): y = h / sqrt(mean h^2 + eps) * weight.  Returns (y, h, rstd): h
    is None without a residual (it is x then), rstd (fp32 [...], for the backward) None
    without ``need_stats``.

    ``weight``: [C], or [groups, C] with one for every one of ``groups`` equal runs of
    consecutive rows (samples, frames), or None.  y has ``out_dtype`` (None: x's; fp32 only
    with x in fp32)."""
    if out is None and _native is not None:
        r = _native.rms_fwd(x, weight, residual, eps, out_dtype, need_stats)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt, rows, C, groups, ptype = _rms_inputs(x, weight, residual)
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in _NORM_TYPES:
        raise TypeError(f"out_dtype must be bfloat16 or float32, got {out_dtype}")
    if out is not None:
        _expect(out, "out", tuple(x.shape), out_dtype)
    _on_device(x, (("weight", weight), ("residual", residual), ("out", out)))
    y = torch.empty(x.shape, dtype=out_dtype, device=x.device) if out is None else out
    h = None if residual is None else torch.empty_like(x)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if need_stats else None
    _no_alias((("out", y),), (("x", x), ("weight", weight), ("residual", residual)))
    _check(library().mw_rmsnorm_fwd(_ptr(x), _ptr(residual), _ptr(weight), _ptr(y), None, _ptr(h), _ptr(rstd),
                                    rows, C, groups, float(eps), xt, _NORM_TYPES[out_dtype], ptype, _stream()))
    return y, h, rstd


def mw_rmsnorm_quantize(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
                        residual: Optional[torch.Tensor] = None, eps: float = 1e-5, need_stats: bool = True):
    """mw_rmsnorm_fwd with y as the product reads it: (q, scale, h, rstd) with y's 8-bit form
    in blocks of (1, 128), as mw_quantize gives it (y itself is not rounded before).  C
    must be a multiple of 16."""
    if _native is not None:
        r = _native.rms_quantize(x, weight, residual, eps, need_stats)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt, rows, C, groups, ptype = _rms_inputs(x, weight, residual)
    _fp8_source(x)
    _on_device(x, (("weight", weight), ("residual", residual)))
    q = torch.empty(x.shape, dtype=_E4M3, device=x.device)
    scale = torch.empty((rows, _blocks(C)), dtype=_E8M0, device=x.device)
    h = None if residual is None else torch.empty_like(x)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if need_stats else None
    _check(library().mw_rmsnorm_fwd(_ptr(x), _ptr(residual), _ptr(weight), _ptr(q), _ptr(scale), _ptr(h),
                                    _ptr(rstd), rows, C, groups, float(eps), xt, 2, ptype, _stream()))
    return q, scale, h, rstd


def mw_rmsnorm_bwd_workspace_size(rows: int, C: int, groups: int) -> int:
    return int(library().mw_rmsnorm_bwd_workspace_size(rows, C, groups))


def mw_rmsnorm_bwd(dy, h, rstd, weight: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None):
    """Gradients (dx, dweight) of sum(y * dy) + sum(h * dh) through mw_rmsnorm_fwd, from its
    h (x where there was no residual) and rstd: dx is the gradient of x and of the residual
    alike; dweight None without a weight."""
    if workspace is None and _native is not None:
        r = _native.rms_bwd(dy, h, rstd, weight, dh)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt, yt = _norm_type(h, "h"), _norm_type(dy, "dy")
    rows, C, groups, ptype = _norm_params(h, weight, None)
    _expect(dy, "dy", tuple(h.shape), dy.dtype)
    if dh is not None:
        _expect(dh, "dh", tuple(h.shape), h.dtype)
    _expect(rstd, "rstd", tuple(h.shape[:-1]), torch.float32)
    _on_device(h, (("dy", dy), ("rstd", rstd), ("weight", weight), ("dh", dh), ("workspace", workspace)))
    ws_bytes = mw_rmsnorm_bwd_workspace_size(rows, C, groups) if weight is not None else 0
    workspace = _workspace(workspace, ws_bytes, h.device)
    dx = torch.empty_like(h)
    dw = None if weight is None else torch.empty_like(weight)
    _no_alias((("workspace", workspace),), (("dy", dy), ("h", h), ("rstd", rstd), ("weight", weight), ("dh", dh)))
    _check(library().mw_rmsnorm_bwd(_ptr(dy), _ptr(h), _ptr(rstd), _ptr(weight), _ptr(dh), _ptr(dx), _ptr(dw),
                                    _ptr(workspace), ws_bytes, rows, C, groups, xt, yt, ptype, _stream()))
    return dx, dw


_FP8_FORMS = {(1, 128): 0, (128, 1): 1, (128, 128): 2}


def _blocks(n: int) -> int:
    return (n + 127) // 128


def _fp8_source(x) -> Tuple[int, int, int]:
    """Type code, rows and columns of a matrix that goes into 8 bits."""
    xt = _norm_type(x, "x")
    if x.dim() < 1 or not x.is_contiguous():
        raise ValueError("x must be a contiguous [..., C] tensor")
    C = x.shape[-1]
    if C % 16:
        raise ValueError(f"x has {C} columns: rows of 8-bit codes must be multiples of 16")
    return xt, math.prod(x.shape[:-1]), C


def mw_quantize(x: torch.Tensor, block: Tuple[int, int] = (1, 128), out=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The 8-bit form of x [..., C] (bf16 or fp32), its rows taken as one matrix [R, C]:
    codes in x's shape (float8_e4m3fn) and for every ``block`` -- (1, 128), (128, 1) or
    (128, 128) elements -- a scale (float8_e8m0fnu), the least power of two s with
    max |x| <= 448 s; x is about code * scale.  Returns (q, scale), scale
    [ceil(R / rows), ceil(C / columns)] for blocks of rows x columns.  A block with a NaN
    or an infinity is NaN.  C must be a multiple of 16.

    ``out`` = (q, scale) reuses caller buffers."""
    if out is None and _native is not None:
        r = _native.quantize(x, block)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt, rows, C = _fp8_source(x)
    form = _FP8_FORMS.get(tuple(block))
    if form is None:
        raise ValueError(f"block must be (1, 128), (128, 1) or (128, 128), got {block}")
    shape = tuple(n if b == 1 else _blocks(n) for n, b in zip((rows, C), block))
    q, scale = out if out is not None else (None, None)
    if out is not None:
        _expect(q, "q", tuple(x.shape), _E4M3)
        _expect(scale, "scale", shape, _E8M0)
    _on_device(x, (("q", q), ("scale", scale)))
    if out is None:
        q = torch.empty(x.shape, dtype=_E4M3, device=x.device)
        scale = torch.empty(shape, dtype=_E8M0, device=x.device)
    else:
        _no_alias((("q", q), ("scale", scale)), (("x", x),))
    outs = (None, None, _ptr(q), _ptr(scale)) if form == 1 else (_ptr(q), _ptr(scale), None, None)
    _check(library().mw_quantize(_ptr(x), *outs, rows, C, form, xt, _stream()))
    return q, scale


def mw_quantize_both(x: torch.Tensor):
    """mw_quantize with blocks of (1, 128) and of (128, 1) elements, x read once:
    (q, scale, q_columns, scale_columns)."""
    if _native is not None:
        r = _native.quantize(x, None)
        if r is not None:
            return r if type(r) is tuple else _check(r)
    xt, rows, C = _fp8_source(x)
    _on_device(x, ())
    q, qc = (torch.empty(x.shape, dtype=_E4M3, device=x.device) for _ in range(2))
    scale, sc = (torch.empty(n, dtype=_E8M0, device=x.device)
                 for n in ((rows, _blocks(C)), (_blocks(rows), C)))
    _check(library().mw_quantize(_ptr(x), _ptr(q), _ptr(scale), _ptr(qc), _ptr(sc), rows, C, 3, xt, _stream()))
    return q, scale, qc, sc


def _fp8_operand(t, scale, name: str, transposed: bool) -> Tuple[int, int, bool]:
    """Rows, contraction and kind of scales (one for 128 rows) of an operand."""
    for v, n, dtype in ((t, name, _E4M3), (scale, f"{name}_scale", _E8M0)):
        if not isinstance(v, torch.Tensor):
            raise TypeError(f"{n} must be a torch.Tensor, got {type(v).__name__}")
        if v.dtype != dtype:
            raise TypeError(f"{n} must be {dtype}, got {v.dtype}")
        if v.dim() != 2 or not v.is_contiguous():
            raise ValueError(f"{n} must be a contiguous matrix")
    if t.shape[1] % 16:
        raise ValueError(f"{name} has {t.shape[1]} columns: rows of 8-bit codes must be multiples of 16")
    rows, K = reversed(t.shape) if transposed else t.shape
    for n, tiles in ((rows, False), (_blocks(rows), True)):
        want = (_blocks(K), n) if transposed else (n, _blocks(K))
        if tuple(scale.shape) == want:
            return rows, K, tiles
    raise ValueError(f"{name}_scale {tuple(scale.shape)} does not fit {name} {tuple(t.shape)}: a scale for "
                     f"every 128 of the contraction, and for every row or 128 of them")


def mw_scaled_matmul(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                     out_dtype: torch.dtype = torch.bfloat16, a_transposed: bool = False,
                     b_transposed: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """c = A B^T of two 8-bit forms, [M, N] in ``out_dtype`` (bf16 or fp32), summed in fp32.

    a: codes [M, K] with scales [M, ceil(K/128)] (blocks of (1, 128)) or [ceil(M/128),
    ceil(K/128)] (of (128, 128)); with ``a_transposed`` codes [K, M] with scales
    [ceil(K/128), M] (blocks of (128, 1)) or [ceil(K/128), ceil(M/128)].  b: the same with
    N in the place of M.  ``out`` reuses a caller's buffer.

    Scales are powers of two (float8_e8m0fnu), as mw_quantize makes them.  A matrix that comes
    with scales of any value (fp32) has to be multiplied out and put into this form.  An fp32
    result sums 8192 of the contraction at most in one tensor-core accumulator, one in bf16
    262144, and longer ones in parts."""
    if out is None and _native is not None:
        r = _native.scaled_matmul(a, a_scale, b, b_scale, out_dtype, a_transposed, b_transposed)
        if r is not None:
            return _check(r) if type(r) is int else r
    M, K, a_tiles = _fp8_operand(a, a_scale, "a", a_transposed)
    N, Kb, b_tiles = _fp8_operand(b, b_scale, "b", b_transposed)
    if K != Kb:
        raise ValueError(f"a has a contraction of {K}, b of {Kb}")
    if out_dtype not in _NORM_TYPES:
        raise TypeError(f"out_dtype must be bfloat16 or float32, got {out_dtype}")
    if out is not None:
        _expect(out, "out", (M, N), out_dtype)
    _on_device(a, (("a_scale", a_scale), ("b", b), ("b_scale", b_scale), ("out", out)))
    c = torch.empty((M, N), dtype=out_dtype, device=a.device) if out is None else out
    _no_alias((("out", c),), (("a", a), ("a_scale", a_scale), ("b", b), ("b_scale", b_scale)))
    _check(library().mw_scaled_matmul(_ptr(a), _ptr(a_scale), int(a_tiles), int(bool(a_transposed)), _ptr(b),
                                      _ptr(b_scale), int(b_tiles), int(bool(b_transposed)), _ptr(c), M, N, K,
                                      _NORM_TYPES[out_dtype], _stream()))
    return c


def mw_device_status(clear: bool = True) -> int:
    """Synchronises the current stream and returns the device status code."""
    return int(library().mw_device_status(_stream(), 1 if clear else 0))


def mw_set_option(name: str, value: int) -> None:
    _check(library().mw_set_option(name.encode(), int(value)))


class RingState:
    """Host-side FIFO bookkeeping of a rolling KV cache (Sec. 3.5).

    ``head`` is the physical row of the logically oldest cached token and
    ``length`` the number of cached tokens.  ``commit(rows)`` returns the
    physical slot where the next ``rows`` tokens are written -- right after
    the newest token -- and evicts the oldest tokens when the ring overflows.
    """

    def __init__(self, cap: int, head: int = 0, length: int = 0):
        if not (cap >= 1 and 0 <= head < cap and 0 <= length <= cap):
            raise ValueError(f"bad ring state cap={cap} head={head} length={length}")
        self.cap, self.head, self.length = cap, head, length

    def commit(self, rows: int) -> int:
        if not 1 <= rows <= self.cap:
            raise ValueError(f"rows={rows} not in [1, {self.cap}]")
        slot = (self.head + self.length) % self.cap
        overflow = max(0, self.length + rows - self.cap)
        self.head = (self.head + overflow) % self.cap
        self.length = min(self.cap, self.length + rows)
        return slot


class _FirstDerivatives(torch.autograd.Function):
    """Gradients that were asked for with a graph of their own: there is no second
    derivative, and without this node it would be left out silently."""

    @staticmethod
    def forward(ctx, what, compute, *inputs):
        ctx.what = what
        return compute(*inputs)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(f"{ctx.what} has no second derivative")


def _first_derivatives(what: str, compute, *inputs):
    """compute(*inputs), the gradients of a function that depend on these tensors."""
    if torch.is_grad_enabled():
        return _FirstDerivatives.apply(what, compute, *inputs)
    return compute(*inputs)


def _aligned_gradient(g: torch.Tensor) -> torch.Tensor:
    """A gradient as 16-byte accesses and copies need it: autograd may deliver a view that
    starts anywhere."""
    g = g.contiguous()
    return g if g.data_ptr() % 16 == 0 else g.clone()


class BlockCausalAttention(torch.autograd.Function):
    """Autograd wrapper: O = block-causal attention(q, k, v) with chunks of T_chunk.  A second
    derivative is refused."""

    @staticmethod
    def forward(ctx, q, k, v, T_chunk: int, scale: Optional[float] = None):
        o, lse = mw_bca_fwd(q, k, v, T_chunk, scale, need_lse=True)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.T_chunk, ctx.scale = T_chunk, scale
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        grads = _first_derivatives(
            "BlockCausalAttention",
            lambda q, k, v, do: mw_bca_bwd(q, k, v, o, lse, do.contiguous(), ctx.T_chunk, ctx.scale), q, k, v, do)
        return (*grads, None, None)


class CrossAttention(torch.autograd.Function):
    """Autograd wrapper: O = cross attention(q, k, v) over the first kv_len states of
    each sample (None: all).  A second derivative is refused."""

    @classmethod
    def apply(cls, q, k, v, kv_len: Optional[torch.Tensor] = None,
              scale: Optional[float] = None):
        if _native is not None:
            r = _native.xattn_apply(q, k, v, kv_len, scale)
            if r is not None:
                return _check(r) if type(r) is int else r
        return super().apply(q, k, v, kv_len, scale)

    @staticmethod
    def forward(ctx, q, k, v, kv_len: Optional[torch.Tensor] = None,
                scale: Optional[float] = None):
        o, lse = mw_xattn_fwd(q, k, v, kv_len, scale, need_lse=True)
        ctx.save_for_backward(q, k, v, o, lse, kv_len)
        ctx.scale = scale
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse, kv_len = ctx.saved_tensors
        grads = _first_derivatives(
            "CrossAttention",
            lambda q, k, v, do: mw_xattn_bwd(q, k, v, o, lse, do.contiguous(), kv_len, ctx.scale), q, k, v, do)
        return (*grads, None, None)


class LayerNorm(torch.autograd.Function):
    """Autograd wrapper: y = layer norm(x) * weight + bias, weight and bias [C], one of
    each for every group of rows ([groups, C]), or None.  A second derivative is refused."""

    @classmethod
    def apply(cls, x, weight: Optional[torch.Tensor] = None,
              bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
              out_dtype: Optional[torch.dtype] = None):
        if _native is not None:
            r = _native.norm_apply(x, weight, bias, eps, out_dtype)
            if r is not None:
                return _check(r) if type(r) is int else r
        return super().apply(x, weight, bias, eps, out_dtype)

    @staticmethod
    def forward(ctx, x, weight: Optional[torch.Tensor] = None,
                bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                out_dtype: Optional[torch.dtype] = None):
        y, mean, rstd = mw_layernorm_fwd(x, weight, bias, eps, out_dtype)
        ctx.save_for_backward(x, weight, bias, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, mean, rstd = ctx.saved_tensors
        grads = _first_derivatives(
            "LayerNorm",
            lambda x, weight, dy: mw_layernorm_bwd(dy.contiguous(), x, mean, rstd, weight, bias), x, weight, dy)
        return (*grads, None, None)


class RMSNorm(torch.autograd.Function):
    """Autograd wrapper: y = RMS norm(x) * weight, weight [C], one for every group of rows
    ([groups, C]), or None; with a residual (y, h) of h = x + residual, through both of which
    gradients come back.  A second derivative is refused."""

    @classmethod
    def apply(cls, x, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
              eps: float = 1e-5, out_dtype: Optional[torch.dtype] = None):
        if _native is not None:
            r = _native.rms_apply(x, weight, residual, eps, out_dtype)
            if r is not None:
                return _check(r) if type(r) is int else r
        return super().apply(x, weight, residual, eps, out_dtype)

    @staticmethod
    def forward(ctx, x, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                eps: float = 1e-5, out_dtype: Optional[torch.dtype] = None):
        y, h, rstd = mw_rmsnorm_fwd(x, weight, residual, eps, out_dtype)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x if h is None else h, weight, rstd)
        ctx.residual, ctx.y_type = residual is not None, y.dtype
        return y if h is None else (y, h)

    @staticmethod
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        if dy is None:  # only h was used
            if dh is None:
                return None, None, None, None, None
            return dh, None, dh, None, None

        def gradients(h, weight, dy, dh):
            return mw_rmsnorm_bwd(dy.contiguous(), h, rstd, weight, None if dh is None else dh.contiguous())

        dx, dw = _first_derivatives("RMSNorm", gradients, h, weight, dy, dh)
        return dx, dw, dx if ctx.residual else None, None, None


class Fp8Linear(torch.autograd.Function):
    """Autograd wrapper: y = x W^T for x [..., K] (bf16 or fp32) and weight [N, K] (bf16 or
    fp32), its three products in 8 bits, in the form of mw_quantize: x and dy in blocks
    along what is summed (a row for y and dx, a column for dW), W in blocks of (128, 128).  y
    has ``out_dtype`` (None: x's); gradients have their inputs' types.  K and N are multiples
    of 16; x and weight start at 16 bytes (gradients may start anywhere).  W's form is made at
    each call: a program whose weights stay keeps mw_quantize(W, (128, 128)) and calls
    mw_scaled_matmul.  A second derivative is refused."""

    @classmethod
    def apply(cls, x, weight, out_dtype: Optional[torch.dtype] = None):
        if _native is not None:
            r = _native.linear_apply(x, weight, out_dtype)
            if r is not None:
                return _check(r) if type(r) is int else r
        return super().apply(x, weight, out_dtype)

    @staticmethod
    def forward(ctx, x, weight, out_dtype: Optional[torch.dtype] = None):
        _norm_type(x, "x")
        _norm_type(weight, "weight")
        if weight.dim() != 2 or x.dim() < 1 or x.shape[-1] != weight.shape[1]:
            raise ValueError(f"x must be [..., K] and weight [N, K], got {tuple(x.shape)} and {tuple(weight.shape)}")
        if weight.shape[0] % 16 or weight.shape[1] % 16 or 0 in weight.shape:
            raise ValueError(f"weight is {tuple(weight.shape)}: N and K must be multiples of 16 above 0")
        x, weight = x.contiguous(), weight.contiguous()
        wq, ws = mw_quantize(weight, (128, 128))
        xc = xcs = None
        if ctx.needs_input_grad[1]:
            xq, xs, xc, xcs = mw_quantize_both(x)
        else:
            xq, xs = mw_quantize(x)
        y = mw_scaled_matmul(xq.view(-1, x.shape[-1]), xs, wq, ws, x.dtype if out_dtype is None else out_dtype)
        ctx.save_for_backward(xc, xcs, wq, ws)
        ctx.types, ctx.shape = (x.dtype, weight.dtype), x.shape
        return y.view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    def backward(ctx, dy):
        xc, xcs, wq, ws = ctx.saved_tensors
        need_x, need_w = ctx.needs_input_grad[:2]
        K = ctx.shape[-1]

        def gradients(dy):
            g = _aligned_gradient(dy).view(-1, wq.shape[0])
            gq = gs = gc = gcs = None
            if need_x and need_w:
                gq, gs, gc, gcs = mw_quantize_both(g)
            elif need_x:
                gq, gs = mw_quantize(g)
            elif need_w:
                gc, gcs = mw_quantize(g, (128, 1))
            dx = dw = None
            if need_x:
                dx = mw_scaled_matmul(gq, gs, wq, ws, ctx.types[0], b_transposed=True).view(ctx.shape)
            if need_w:
                dw = mw_scaled_matmul(gc, gcs, xc.view(-1, K), xcs, ctx.types[1], a_transposed=True, b_transposed=True)
            return dx, dw

        # (what the gradients depend on besides is saved in 8 bits, without its graph: any
        # input that wants a gradient stands for it)
        stand_in = torch.empty(0, requires_grad=True) if torch.is_grad_enabled() else None
        return (*_first_derivatives("Fp8Linear", lambda dy, _: gradients(dy), dy, stand_in), None)
