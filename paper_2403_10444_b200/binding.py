"""ctypes binding of libbv_b200.so: argument marshalling only.

Every step of the verification path runs inside the CUDA library; nothing here
computes.  There is no CPU fallback: if the library is missing, or an entry
point reports an error, an exception is raised.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from typing import Optional, Tuple

import torch

try:
    from . import _fast          # the cache's calls marshalled in C++ (build.build_fast); without it they are marshalled below
except ImportError:
    _fast = None

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libbv_b200.so")

DTYPE_F32 = 0
DTYPE_BF16 = 1

# every symbol include/bv.h declares
EXPORTS = ["bv_verify", "tv_verify", "bv_verify_ex", "tv_verify_ex", "bv_verify_host",
           "tv_verify_host", "bv_verify_noalloc", "bv_verify_lse", "bv_verify_lse_ex", "tv_verify_lse", "tv_verify_lse_ex", "gbv_verify", "gbv_verify_ex", "bv_verify_probs", "tv_verify_probs", "bv_sample_draft", "bv_draft_chain", "bv_decode_loop", "bv_cache_attend", "bv_cache_append", "bv_pages_extend", "bv_pages_truncate", "bv_pages_fork", "bv_pages_compact", "bv_pages_copy", "bv_cache_append_rotary", "bv_prompt_attend", "bv_sample_filtered", "bv_stream_status", "bv_set_option", "bv_release", "bv_last_launch_count", "bv_last_kernel", "bv_last_cuda_error",
           "bv_status_string", "bv_version"]


class BVError(RuntimeError):
    """An entry point of libbv_b200.so returned a non-zero status."""

    def __init__(self, status: int, text: str):
        super().__init__("libbv_b200: %s (status %d)" % (text, status))
        self.status = status


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libbv_b200.so (built by ``python -m paper_2403_10444_b200.build``)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or _LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(
            "CUDA library %s is missing: build it with `python -m paper_2403_10444_b200.build` "
            "(there is no CPU fallback)" % p)
    lib = ctypes.CDLL(p)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    base = [vp, vp, vp, vp, ci, ci, ci, ci, cf, vp, vp]
    for name in ("bv_verify", "tv_verify", "bv_verify_noalloc", "gbv_verify"):
        getattr(lib, name).argtypes = base + [vp]
    for name in ("bv_verify_ex", "tv_verify_ex", "gbv_verify_ex"):
        getattr(lib, name).argtypes = base + [vp, vp, vp, vp, vp, vp]
    for name in ("bv_verify_host", "tv_verify_host"):
        getattr(lib, name).argtypes = base
    lib.bv_sample_draft.argtypes = [vp, vp, ci, ci, ci, cf, vp, vp, vp]
    lib.bv_draft_chain.argtypes = [vp, vp, vp, ci, ci, ci, ci, cf, vp, vp, vp]
    lib.bv_decode_loop.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, ci, vp, vp, vp, vp, vp, vp, vp]
    for name in ("bv_verify_probs", "tv_verify_probs"):
        getattr(lib, name).argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp]
    for name in ("bv_verify_lse", "tv_verify_lse"):
        getattr(lib, name).argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, cf, vp, vp, vp]
        getattr(lib, name + "_ex").argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, cf, vp, vp, vp, vp, vp, vp, vp, vp]
    # (bv_cache and the strides travel as packed bytes)
    lib.bv_cache_attend.argtypes = [vp, vp, vp, vp, ci, ci, cf, ci, ci, vp, vp, vp]
    lib.bv_cache_append.argtypes = [vp, vp, vp, vp, vp, vp, ci, vp]
    lib.bv_pages_extend.argtypes = [vp, vp, ci, vp, vp, vp]
    lib.bv_pages_truncate.argtypes = [vp, vp, vp, ci, vp]
    lib.bv_pages_fork.argtypes = [vp, vp, vp, ci, vp, vp]
    lib.bv_pages_compact.argtypes = [vp, vp, vp, vp]
    lib.bv_pages_copy.argtypes = [vp, vp, ci, vp, vp]
    lib.bv_cache_append_rotary.argtypes = [vp, vp, vp, vp, ci, vp, vp, vp, vp, vp, vp, ci, vp, vp, vp, vp, vp]
    lib.bv_prompt_attend.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, ci, vp, vp, vp]
    lib.bv_sample_filtered.argtypes = [vp, ctypes.c_int64, vp, ci, ci, ci, vp, vp, vp, vp, ctypes.c_int64, vp]
    for name in EXPORTS:
        getattr(lib, name).restype = ci
    lib.bv_stream_status.argtypes = [vp]
    lib.bv_set_option.argtypes = [ctypes.c_char_p, ci]
    lib.bv_status_string.restype = ctypes.c_char_p
    lib.bv_status_string.argtypes = [ci]
    if path is None:
        _lib = lib
        if _fast is not None:
            _fast.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in
                         ("bv_cache_attend", "bv_cache_append", "bv_pages_extend", "bv_pages_truncate", "bv_pages_fork", "bv_pages_compact", "bv_pages_copy",
                          "bv_cache_append_rotary", "bv_prompt_attend", "bv_sample_filtered")))
    return lib


def bv_status_string(status: int) -> str:
    return load_library().bv_status_string(int(status)).decode()


def bv_version() -> int:
    return int(load_library().bv_version())


def bv_last_launch_count() -> int:
    return int(load_library().bv_last_launch_count())


def bv_last_kernel() -> int:
    """Code of the kernel the last verification call on this thread launched (1 flow, 2 cluster,
    3 element-wise streaming, 4 small-batch, 5 phase)."""
    return int(load_library().bv_last_kernel())


def bv_release() -> None:
    _check(load_library().bv_release())


def bv_set_option(name: str, value: int) -> None:
    """Process-wide tuning / test option of the library (see include/bv.h); 0 restores the default."""
    _check(load_library().bv_set_option(name.encode(), int(value)))


def bv_stream_status(stream=None) -> int:
    """Waits for the stream and returns 0, or -4 if a device-side wait of a call on it gave up."""
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(load_library().bv_stream_status(ctypes.c_void_p(s.cuda_stream)))


def _check(status: int) -> None:
    if status != 0:
        lib = load_library()
        text = lib.bv_status_string(int(status)).decode()
        if status == -3:
            text += " (cudaError %d)" % lib.bv_last_cuda_error()
        raise BVError(status, text)


class _Nothing:
    def __enter__(self):
        return None

    def __exit__(self, *exc):
        return False


_NOTHING = _Nothing()


def _on(dev: torch.device):
    """The context in which ``dev`` is the current device (nothing to enter if it is already: entering costs 1.4 us of host
    time)."""
    return _NOTHING if dev.index == torch.cuda.current_device() else torch.cuda.device(dev)


def _raw_stream(dev: torch.device, stream) -> int:
    """The cudaStream_t of ``stream``, or of torch's current stream on ``dev`` (without the Stream object around it: 2 us)."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev.index)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return DTYPE_F32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    raise TypeError("logits must be float32 or bfloat16, got %s" % t.dtype)


def _shapes(target, draft, tokens, uniforms, want_cuda: bool):
    if target.dim() != 3 or draft.dim() != 3:
        raise ValueError("target_logits must be [B, gamma+1, V] and draft_logits [B, gamma, V]")
    B, g1, V = target.shape
    gamma = g1 - 1
    if draft.shape != (B, gamma, V):
        raise ValueError("draft_logits must be [B, gamma, V]")
    if tokens.shape != (B, gamma) or tokens.dtype != torch.int32:
        raise ValueError("draft_tokens must be int32 [B, gamma]")
    if uniforms.shape != (B, gamma + 2) or uniforms.dtype != torch.float32:
        raise ValueError("uniforms must be float32 [B, gamma+2]")
    if target.dtype != draft.dtype:
        raise TypeError("target and draft logits must share a dtype")
    if not (target.is_contiguous() and draft.is_contiguous() and tokens.is_contiguous() and uniforms.is_contiguous()):
        raise ValueError("all tensors must be contiguous")
    if not (target.is_cuda == draft.is_cuda == tokens.is_cuda == uniforms.is_cuda == want_cuda):
        raise ValueError("expected %s tensors" % ("CUDA" if want_cuda else "host"))
    return B, gamma, V


def _device_call(name: str, target, draft, tokens, uniforms, temperature, diagnostics: bool,
                 stream: Optional[torch.cuda.Stream]):
    lib = load_library()
    B, gamma, V = _shapes(target, draft, tokens, uniforms, True)
    dev = target.device
    out_tokens, out_len = target.new_empty((B, gamma + 1), dtype=torch.int32), target.new_empty((B,), dtype=torch.int32)
    with _on(dev):
        s = _raw_stream(dev, stream)
        args = [target.data_ptr(), draft.data_ptr(), tokens.data_ptr(), uniforms.data_ptr(),
                B, gamma, V, _dtype_code(target), float(temperature),
                out_tokens.data_ptr(), out_len.data_ptr()]
        if diagnostics:
            f = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)
            diag = dict(p=f(B, gamma + 1), S=f(B, gamma), h=f(B, gamma + 1),
                        lse_t=f(B, gamma + 1), lse_d=f(B, gamma))
            args += [diag[k].data_ptr() for k in ("p", "S", "h", "lse_t", "lse_d")]
        _check(getattr(lib, name)(*args, s))
    if diagnostics:
        return out_tokens, out_len, diag
    return out_tokens, out_len


def bv_verify(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
              stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Block Verification (Algorithm 2) on CUDA tensors; returns (out_tokens, out_len)."""
    return _device_call("bv_verify", target_logits, draft_logits, draft_tokens, uniforms,
                        temperature, False, stream)


def tv_verify(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
              stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Token Verification (Algorithm 1) on CUDA tensors; returns (out_tokens, out_len)."""
    return _device_call("tv_verify", target_logits, draft_logits, draft_tokens, uniforms,
                        temperature, False, stream)


def bv_verify_ex(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
                 stream=None):
    """bv_verify plus its intermediates: returns (out_tokens, out_len, dict(p, S, h, lse_t, lse_d))."""
    return _device_call("bv_verify_ex", target_logits, draft_logits, draft_tokens, uniforms,
                        temperature, True, stream)


def tv_verify_ex(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
                 stream=None):
    """tv_verify plus its intermediates (NaN where Algorithm 1 forms none)."""
    return _device_call("tv_verify_ex", target_logits, draft_logits, draft_tokens, uniforms,
                        temperature, True, stream)


def gbv_verify(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
               stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Greedy Block Verification, one iteration (Algorithm 4), on CUDA tensors; returns
    (out_tokens, out_len).  Rows must be whole 16-byte vectors."""
    return _device_call("gbv_verify", target_logits, draft_logits, draft_tokens, uniforms,
                        temperature, False, stream)


def gbv_verify_ex(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
                  stream=None):
    """gbv_verify plus its intermediates: p holds the unclipped products, S the numerator sums of
    the acceptance ratios, h the ratios (above one, or +inf, where the test passes with certainty)."""
    return _device_call("gbv_verify_ex", target_logits, draft_logits, draft_tokens, uniforms,
                        temperature, True, stream)


def _probs_call(name: str, target_probs, draft_probs, tokens, uniforms, diagnostics: bool, stream):
    lib = load_library()
    B, gamma, V = _shapes(target_probs, draft_probs, tokens, uniforms, True)
    dev = target_probs.device
    out_tokens, out_len = target_probs.new_empty((B, gamma + 1), dtype=torch.int32), target_probs.new_empty((B,), dtype=torch.int32)
    diag, ptrs = None, [None, None, None]
    if diagnostics:
        f = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)
        diag = dict(p=f(B, gamma + 1), S=f(B, gamma), h=f(B, gamma + 1))
        ptrs = [diag[k].data_ptr() for k in ("p", "S", "h")]
    with _on(dev):
        s = _raw_stream(dev, stream)
        _check(getattr(lib, name)(target_probs.data_ptr(), draft_probs.data_ptr(), tokens.data_ptr(),
                                  uniforms.data_ptr(), B, gamma, V, _dtype_code(target_probs),
                                  out_tokens.data_ptr(), out_len.data_ptr(), *ptrs, s))
    return (out_tokens, out_len, diag) if diagnostics else (out_tokens, out_len)


def bv_verify_probs(target_probs, draft_probs, draft_tokens, uniforms, diagnostics: bool = False, stream=None):
    """Block Verification (Algorithm 2) on given probabilities [B, gamma+1, V] / [B, gamma, V] (CUDA,
    float32 or bfloat16, used as stored); returns (out_tokens, out_len) and, with ``diagnostics``,
    dict(p, S, h)."""
    return _probs_call("bv_verify_probs", target_probs, draft_probs, draft_tokens, uniforms, diagnostics, stream)


def tv_verify_probs(target_probs, draft_probs, draft_tokens, uniforms, diagnostics: bool = False, stream=None):
    """Token Verification (Algorithm 1) on given probabilities; see bv_verify_probs."""
    return _probs_call("tv_verify_probs", target_probs, draft_probs, draft_tokens, uniforms, diagnostics, stream)


def bv_verify_noalloc(target_logits, draft_logits, draft_tokens, uniforms, out_tokens, out_len,
                      temperature: float = 1.0, stream=None) -> None:
    """Block Verification through the entry point that allocates nothing.

    For embedders that cannot let the library allocate device memory when they call it
    (a memory pool that owns the device, possible stream capture, allocator hooks).  The
    caller supplies the outputs: ``out_tokens`` int32 [B, gamma+1] and ``out_len`` int32 [B],
    CUDA tensors; this wrapper creates no tensor either.  Raises BVError(status -5) when the
    problem needs more than the library's fixed 8 MiB scratch array.
    """
    lib = load_library()
    B, gamma, V = _shapes(target_logits, draft_logits, draft_tokens, uniforms, True)
    if tuple(out_tokens.shape) != (B, gamma + 1) or out_tokens.dtype != torch.int32 or not out_tokens.is_cuda:
        raise ValueError("out_tokens must be a CUDA int32 tensor [B, gamma+1]")
    if tuple(out_len.shape) != (B,) or out_len.dtype != torch.int32 or not out_len.is_cuda:
        raise ValueError("out_len must be a CUDA int32 tensor [B]")
    dev = target_logits.device
    with _on(dev):
        s = _raw_stream(dev, stream)
        _check(lib.bv_verify_noalloc(target_logits.data_ptr(), draft_logits.data_ptr(),
                                     draft_tokens.data_ptr(), uniforms.data_ptr(), B, gamma, V,
                                     _dtype_code(target_logits), float(temperature),
                                     out_tokens.data_ptr(), out_len.data_ptr(), s))


def _host_call(name: str, target, draft, tokens, uniforms, temperature, out_tokens, out_len):
    lib = load_library()
    B, gamma, V = _shapes(target, draft, tokens, uniforms, False)
    if out_tokens is None:
        out_tokens = torch.empty((B, gamma + 1), dtype=torch.int32).pin_memory()
    if out_len is None:
        out_len = torch.empty((B,), dtype=torch.int32).pin_memory()
    _check(getattr(lib, name)(target.data_ptr(), draft.data_ptr(), tokens.data_ptr(),
                              uniforms.data_ptr(), B, gamma, V, _dtype_code(target),
                              float(temperature), out_tokens.data_ptr(), out_len.data_ptr()))
    return out_tokens, out_len


def bv_verify_host(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
                   out_tokens=None, out_len=None):
    """Block Verification on HOST tensors (pinned for speed): copies in, runs, copies out."""
    return _host_call("bv_verify_host", target_logits, draft_logits, draft_tokens, uniforms,
                      temperature, out_tokens, out_len)


def tv_verify_host(target_logits, draft_logits, draft_tokens, uniforms, temperature: float = 1.0,
                   out_tokens=None, out_len=None):
    """Token Verification on HOST tensors (pinned for speed): copies in, runs, copies out."""
    return _host_call("tv_verify_host", target_logits, draft_logits, draft_tokens, uniforms,
                      temperature, out_tokens, out_len)


def bv_sample_draft(logits, uniforms, temperature: float = 1.0, want_lse: bool = True, stream=None):
    """The drafting step of Algorithm 3 on CUDA tensors: logits [rows, V] (float32 or bfloat16),
    uniforms [rows] float32.  Returns (tokens int32 [rows], lse float32 [rows] or None)."""
    if not (logits.is_cuda and uniforms.is_cuda):
        raise ValueError("bv_sample_draft takes CUDA tensors")
    if logits.dim() != 2 or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous [rows, V] tensor")
    rows, V = logits.shape
    if uniforms.shape != (rows,) or uniforms.dtype != torch.float32 or not uniforms.is_contiguous():
        raise ValueError("uniforms must be a contiguous float32 tensor of [rows]")
    lib = load_library()
    tokens = torch.empty((rows,), dtype=torch.int32, device=logits.device)
    lse = torch.empty((rows,), dtype=torch.float32, device=logits.device) if want_lse else None
    dev = logits.device
    with _on(dev):
        _check(lib.bv_sample_draft(logits.data_ptr(), uniforms.data_ptr(), rows, V, _dtype_code(logits),
                                   float(temperature), tokens.data_ptr(), lse.data_ptr() if want_lse else None,
                                   _raw_stream(dev, stream)))
    return tokens, lse


def bv_draft_chain(draft_table, first_tokens, uniforms, temperature: float = 1.0, stream=None):
    """The whole drafting step for a last-token table model: draft_table CUDA [V, V] float32 or bfloat16,
    first_tokens CUDA int32 [B], uniforms CUDA float32 [gamma, B]; returns (tokens int32 [B, gamma],
    lse float32 [B, gamma]) from one launch."""
    lib = load_library()
    V = draft_table.shape[0]
    if draft_table.dim() != 2 or draft_table.shape[1] != V or not draft_table.is_cuda or not draft_table.is_contiguous():
        raise ValueError("draft_table must be a contiguous CUDA tensor [V, V]")
    B = first_tokens.shape[0]
    if first_tokens.dtype != torch.int32 or not first_tokens.is_cuda or not first_tokens.is_contiguous() or first_tokens.dim() != 1:
        raise ValueError("first_tokens must be a contiguous CUDA int32 tensor [B]")
    if (uniforms.dim() != 2 or uniforms.shape[1] != B or uniforms.dtype != torch.float32 or not uniforms.is_cuda
            or not uniforms.is_contiguous()):
        raise ValueError("uniforms must be a contiguous CUDA float32 tensor [gamma, B]")
    gamma = uniforms.shape[0]
    dev = draft_table.device
    tokens = torch.empty((B, gamma), dtype=torch.int32, device=dev)
    lse = torch.empty((B, gamma), dtype=torch.float32, device=dev)
    with _on(dev):
        s = _raw_stream(dev, stream)
        _check(lib.bv_draft_chain(draft_table.data_ptr(), first_tokens.data_ptr(), uniforms.data_ptr(), B, gamma, V,
                                  _dtype_code(draft_table), float(temperature), tokens.data_ptr(), lse.data_ptr(),
                                  s))
    return tokens, lse


def bv_decode_loop(target_table, draft_table, first_tokens, u_draft, u_verify, gamma: int, temperature: float, algo: int):
    """The decoding loop for two last-token table models (see include/bv.h; contiguous CUDA tensors, all checked, algo as there): (tokens,
    lengths, tau, drafted, fault), or None where the library has no kernel for the call."""
    V = target_table.shape[0]
    if target_table.shape != (V, V) or draft_table.shape != (V, V) or target_table.dtype != draft_table.dtype:
        raise ValueError("the model tables must be [V, V] of one dtype")
    if first_tokens.dim() != 1 or first_tokens.dtype != torch.int32:
        raise ValueError("first_tokens must be int32 [B]")
    N, B = u_draft.shape[0], first_tokens.shape[0]
    if u_draft.shape != (N, gamma, B) or u_verify.shape != (N, B, gamma + 2) or u_draft.dtype != torch.float32 or u_verify.dtype != torch.float32:
        raise ValueError("u_draft must be float32 [N, gamma, B] and u_verify float32 [N, B, gamma+2]")
    if not (target_table.is_contiguous() and draft_table.is_contiguous() and first_tokens.is_contiguous() and u_draft.is_contiguous() and u_verify.is_contiguous()):
        raise ValueError("all tensors must be contiguous")
    if not (0 <= target_table.get_device() == draft_table.get_device() == first_tokens.get_device() == u_draft.get_device() == u_verify.get_device()):
        raise ValueError("expected CUDA tensors on one device")
    lib = load_library()
    dev = target_table.device
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)
    tokens, tau, drafted, fault = i32(B, N * (gamma + 1)), i32(N, B), i32(N, B, gamma), i32(1)
    lengths = torch.empty((B,), dtype=torch.int64, device=dev)
    work = i32(B * (2 * gamma + 3))
    with _on(dev):
        status = lib.bv_decode_loop(target_table.data_ptr(), draft_table.data_ptr(), first_tokens.data_ptr(), u_draft.data_ptr(),
                                    u_verify.data_ptr(), N, B, gamma, V, _dtype_code(target_table), float(temperature), algo,
                                    tokens.data_ptr(), lengths.data_ptr(), tau.data_ptr(), drafted.data_ptr(), fault.data_ptr(),
                                    work.data_ptr(), _raw_stream(dev, None))
    if status == -2:
        return None
    _check(status)
    return tokens, lengths, tau, drafted, fault


def bv_verify_lse(target_logits, draft_logits, draft_tokens, uniforms, draft_lse, temperature: float = 1.0,
                  diagnostics: bool = False, stream=None):
    """Block Verification with the draft rows' log-normalisers supplied (float32 CUDA tensor
    [B, gamma], e.g. the second output of bv_sample_draft reshaped).  Returns (out_tokens, out_len)
    or, with ``diagnostics``, (out_tokens, out_len, dict of p, S, h, lse_t, lse_d)."""
    return _lse_call("bv_verify_lse", target_logits, draft_logits, draft_tokens, uniforms, draft_lse, temperature,
                     diagnostics, stream)


def tv_verify_lse(target_logits, draft_logits, draft_tokens, uniforms, draft_lse, temperature: float = 1.0,
                  diagnostics: bool = False, stream=None):
    """Token Verification with the draft rows' log-normalisers supplied; see bv_verify_lse."""
    return _lse_call("tv_verify_lse", target_logits, draft_logits, draft_tokens, uniforms, draft_lse, temperature,
                     diagnostics, stream)


def _lse_call(name, target_logits, draft_logits, draft_tokens, uniforms, draft_lse, temperature, diagnostics, stream):
    lib = load_library()
    B, gamma, V = _shapes(target_logits, draft_logits, draft_tokens, uniforms, True)
    if (not draft_lse.is_cuda or draft_lse.dtype != torch.float32 or tuple(draft_lse.shape) != (B, gamma)
            or not draft_lse.is_contiguous()):
        raise ValueError("draft_lse must be a contiguous float32 CUDA tensor of [B, gamma]")
    dev = target_logits.device
    out_tokens, out_len = target_logits.new_empty((B, gamma + 1), dtype=torch.int32), target_logits.new_empty((B,), dtype=torch.int32)
    with _on(dev):
        s = _raw_stream(dev, stream)
        args = [target_logits.data_ptr(), draft_logits.data_ptr(), draft_tokens.data_ptr(), uniforms.data_ptr(),
                draft_lse.data_ptr(), B, gamma, V, _dtype_code(target_logits), float(temperature),
                out_tokens.data_ptr(), out_len.data_ptr()]
        if diagnostics:
            f = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)
            diag = dict(p=f(B, gamma + 1), S=f(B, gamma), h=f(B, gamma + 1), lse_t=f(B, gamma + 1), lse_d=f(B, gamma))
            args += [diag[k].data_ptr() for k in ("p", "S", "h", "lse_t", "lse_d")]
            _check(getattr(lib, name + "_ex")(*args, s))
            return out_tokens, out_len, diag
        _check(getattr(lib, name)(*args, s))
    return out_tokens, out_len


# ---- the paged key-value cache (include/bv.h, struct bv_cache) ----
#
# A call of the cache takes some 10 us on the GPU and is made for every layer.  What is in order goes through _fast (5 us of host time a
# call, nearly all of it the launch); what it will not take, and everything where it is not built, is checked here, where what
# a check finds wrong is put in words (7 us more).

_CACHE = struct.Struct("@5Q6q8i")
_STRIDES = struct.Struct("@3q")
_I32 = torch.int32
_CODES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _enqueue(fn, dev: int, *args) -> None:
    """Calls an entry point with device ``dev`` current (it nearly always is) and its current stream as the last argument."""
    if torch._C._cuda_getDevice() == dev:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if status:
        _check(status)


def _on_stream(stream, of, fn, *args):
    """A call on a stream that is given: what it allocates and fills belongs to that stream too."""
    if stream.device != of.device:
        raise ValueError("the stream must be one of the cache's device")
    with torch.cuda.stream(stream):
        return fn(*args)


def _pools(k, v):
    """(shape, strides of k, strides of v, dtype code, dtype, device) of two pools of pages [num_pages, heads, page_size, D]."""
    shape, ks, vs, dtype, dev = k.shape, k.stride(), v.stride(), k.dtype, k.get_device()
    if len(shape) != 4 or ks[3] != 1 or len(vs) != 4 or vs[3] != 1:
        raise ValueError("k and v must be [num_pages, heads, page_size, D] with contiguous rows of D")
    if v.shape != shape or v.dtype is not dtype:
        raise ValueError("k and v must have one shape and dtype")
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError("keys and values must be float32 or bfloat16, got %s" % dtype)
    return shape, ks, vs, code, dtype, dev


def _table(table, lens):
    """(B, width, device) of a table of pages and its lengths."""
    shape, dev = table.shape, table.get_device()
    if len(shape) != 2 or lens.shape != shape[:1] or table.dtype is not _I32 or lens.dtype is not _I32:
        raise ValueError("table must be int32 [B, width] and lens int32 [B]")
    if not (table.is_contiguous() and lens.is_contiguous()):
        raise ValueError("table and lens must be contiguous")
    if dev < 0 or lens.get_device() != dev:
        raise ValueError("expected CUDA tensors on one device")
    return shape[0], shape[1], dev


def _written(t, name: str) -> None:
    """A tensor that is written must not have two elements in one place."""
    if not t.is_contiguous() and any(st == 0 and n > 1 for st, n in zip(t.stride(), t.shape)):
        raise ValueError("%s must not be an expanded tensor" % name)


def _counted(t, n: int, dev: int, name: str):
    """Address of an int32 [n] on the cache's device (None: null)."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError("%s must be a contiguous int32 tensor [%d] on the cache's device" % (name, n))
    return t.data_ptr()


def _cache(k, v, table, lens):
    """The packed cache, its B, heads, D, dtype and device."""
    (P, heads, page, D), ks, vs, code, dtype, dev = _pools(k, v)
    B, width, on = _table(table, lens)
    if dev != on or v.get_device() != on:
        raise ValueError("expected CUDA tensors on one device")
    return _CACHE.pack(k.data_ptr(), v.data_ptr(), table.data_ptr(), lens.data_ptr(), 0, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                       B, width, P, page, heads, D, code, 0), B, heads, D, dtype, dev


def _rows(t, B: int, heads: int, D: int, dtype, dev: int, name: str):
    """(n, heads, packed strides) of a tensor [B, n, heads, D] that goes with the cache (heads = 0: any number)."""
    shape, st = t.shape, t.stride()
    if len(shape) != 4 or shape[0] != B or shape[3] != D or (heads and shape[2] != heads) or t.dtype is not dtype:
        raise ValueError("%s must be [B, n, heads, D] of the cache's dtype" % name)
    if st[3] != 1 or t.get_device() != dev:
        raise ValueError("%s must have contiguous rows of D on the cache's device" % name)
    return shape[1], shape[2], _STRIDES.pack(st[0], st[1], st[2])


def bv_cache_attend(q, k, v, table, lens, n_new=None, scale: Optional[float] = None, window: int = 0, sinks: int = 0, out=None,
                    stream=None):
    """Attention of the newest tokens of each sequence over a paged key-value cache (see include/bv.h).

    ``q`` [B, n, q_heads, D]; ``k``, ``v`` [num_pages, heads, page_size, D] (float32 or bfloat16, any strides with contiguous rows);
    ``table`` int32 [B, width], ``lens`` int32 [B] (the newest tokens counted in), ``n_new`` int32 [B] or None: every sequence
    brings n.  ``scale``: 1/sqrt(D) by default; ``window`` > 0: a token sees its last ``window`` positions and the first ``sinks``.
    Returns ``out`` [B, n, q_heads, D] (rows beyond n_new[b] are not written: zero in a tensor made here).  Forward only: what is returned has no
    autograd graph, whether or not ``q``, ``k`` or ``v`` require gradients."""
    if stream is not None:
        return _on_stream(stream, lens, bv_cache_attend, q, k, v, table, lens, n_new, scale, window, sinks, out)
    if _fast is not None:
        r = _fast.attend(q, k, v, table, lens, n_new, scale, window, sinks, out)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, B, _, D, dtype, dev = _cache(k, v, table, lens)
    n, heads, qs = _rows(q, B, 0, D, dtype, dev, "q")
    if out is None:
        out = q.new_empty((B, n, heads, D)) if n_new is None else q.new_zeros((B, n, heads, D))
    else:
        _written(out, "out")
    n_out, _, os_ = _rows(out, B, heads, D, dtype, dev, "out")
    if n_out != n:
        raise ValueError("out must have the shape of q")
    new = None if n_new is None else _counted(n_new, B, dev, "n_new")
    if B == 0:
        return out
    _enqueue((_lib or load_library()).bv_cache_attend, dev, blob, q.data_ptr(), qs, new, n, heads, D ** -0.5 if scale is None else scale, window, sinks, out.data_ptr(), os_)
    return out


def bv_cache_append(k_new, v_new, k, v, table, lens, n_new=None, stream=None) -> None:
    """Stores the keys and values of the newest tokens [B, n, heads, D] in the pages of their positions (see include/bv.h); autograd does not see it."""
    if stream is not None:
        return _on_stream(stream, lens, bv_cache_append, k_new, v_new, k, v, table, lens, n_new)
    if _fast is not None:
        r = _fast.append(k_new, v_new, k, v, table, lens, n_new)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, B, heads, D, dtype, dev = _cache(k, v, table, lens)
    n, _, ks = _rows(k_new, B, heads, D, dtype, dev, "k_new")
    n_v, _, vs = _rows(v_new, B, heads, D, dtype, dev, "v_new")
    if n != n_v:
        raise ValueError("k_new and v_new must have one shape")
    _written(k, "k")
    _written(v, "v")
    new = None if n_new is None else _counted(n_new, B, dev, "n_new")
    if B == 0:
        return
    _enqueue((_lib or load_library()).bv_cache_append, dev, blob, k_new.data_ptr(), ks, v_new.data_ptr(), vs, new, n)


def _book(table, lens, refs, page_size: int):
    """The packed cache of a call that moves no keys, B and device."""
    B, width, dev = _table(table, lens)
    if refs.dtype is not _I32 or refs.dim() != 1 or not refs.is_contiguous() or refs.get_device() != dev:
        raise ValueError("refs must be a contiguous int32 tensor [num_pages] on the table's device")
    return _CACHE.pack(0, 0, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), 0, 0, 0, 0, 0, 0, B, width, refs.shape[0], page_size, 0, 0, 0, 0), B, dev


def bv_pages_extend(table, lens, refs, page_size: int, n: int, n_new=None, stream=None):
    """Lengthens every sequence by n (or n_new[b] in 0 .. n) tokens, taking the lowest free pages (refs 0) in the sequences' order; table, lens and
    refs change in place.  Returns (new int32 [B]: the tokens, or -1 for a sequence left as it was; copies int32 [B, 2]: the pages that
    bv_pages_copy is to copy, or -1)."""
    if stream is not None:
        return _on_stream(stream, lens, bv_pages_extend, table, lens, refs, page_size, n, n_new)
    if _fast is not None:
        r = _fast.extend(table, lens, refs, page_size, n, n_new)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, B, dev = _book(table, lens, refs, page_size)
    given = None if n_new is None else _counted(n_new, B, dev, "n_new")
    new, copies = table.new_empty((B,)), table.new_empty((B, 2))
    if B == 0:
        return new, copies
    _enqueue((_lib or load_library()).bv_pages_extend, dev, blob, given, n, new.data_ptr(), copies.data_ptr())
    return new, copies


def bv_pages_truncate(table, lens, refs, page_size: int, keep, n: int = 0, n_new=None, stream=None) -> None:
    """Keeps the first keep[b] of the n (or n_new[b]) newest tokens of each sequence, with n = 0 of all its tokens, and gives back the pages
    that hold nothing any more.  ``keep`` may be the out_len of a verification."""
    if stream is not None:
        return _on_stream(stream, lens, bv_pages_truncate, table, lens, refs, page_size, keep, n, n_new)
    if _fast is not None:
        r = _fast.truncate(table, lens, refs, page_size, keep, n, n_new)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, B, dev = _book(table, lens, refs, page_size)
    kept, given = _counted(keep, B, dev, "keep"), None if n_new is None else _counted(n_new, B, dev, "n_new")
    if B == 0:
        return
    _enqueue((_lib or load_library()).bv_pages_truncate, dev, blob, kept, given, n)


def bv_pages_fork(table, lens, refs, page_size: int, src, dst, stream=None):
    """Makes sequence dst[i] a second copy of src[i] on the same pages.  Returns ok int32: 0, or -1 where a fork is refused."""
    if stream is not None:
        return _on_stream(stream, lens, bv_pages_fork, table, lens, refs, page_size, src, dst)
    if _fast is not None:
        r = _fast.fork(table, lens, refs, page_size, src, dst)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, _, dev = _book(table, lens, refs, page_size)
    forks = src.shape[0] if src.dim() == 1 else -1
    s, d = _counted(src, forks, dev, "src"), _counted(dst, forks, dev, "dst")
    ok = table.new_empty((forks,))
    if forks == 0:
        return ok
    _enqueue((_lib or load_library()).bv_pages_fork, dev, blob, s, d, forks, ok.data_ptr())
    return ok


def bv_pages_compact(table, lens, refs, page_size: int, stream=None):
    """Renumbers the pages so that those in use come first.  Returns (moves int32 [num_pages // 2, 2], count int32 [1]), which
    bv_pages_copy takes for each layer before anything else uses the cache."""
    if stream is not None:
        return _on_stream(stream, lens, bv_pages_compact, table, lens, refs, page_size)
    if _fast is not None:
        r = _fast.compact(table, lens, refs, page_size)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, _, dev = _book(table, lens, refs, page_size)
    moves, count = table.new_empty((refs.shape[0] // 2, 2)), table.new_empty((1,))
    # (a pool of one page has no moves, and no place for them)
    _enqueue((_lib or load_library()).bv_pages_compact, dev, blob, moves.data_ptr() or count.data_ptr(), count.data_ptr())
    return moves, count


def bv_pages_copy(k, v, pairs, count=None, stream=None) -> None:
    """Copies pages, keys and values: pairs int32 [n, 2] of source and destination, of which the first count[0] are looked at."""
    if stream is not None:
        return _on_stream(stream, k, bv_pages_copy, k, v, pairs, count)
    if _fast is not None:
        r = _fast.copy(k, v, pairs, count)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    (P, heads, page, D), ks, vs, code, _, dev = _pools(k, v)
    _written(k, "k")
    _written(v, "v")
    if dev < 0 or v.get_device() != dev:
        raise ValueError("expected CUDA tensors on one device")
    shape = pairs.shape
    if pairs.dtype is not _I32 or len(shape) != 2 or shape[1] != 2 or not pairs.is_contiguous() or pairs.get_device() != dev:
        raise ValueError("pairs must be a contiguous int32 tensor [n, 2] on the cache's device")
    upto = None if count is None else _counted(count, 1, dev, "count")
    if shape[0] == 0:
        return
    blob = _CACHE.pack(k.data_ptr(), v.data_ptr(), 0, 0, 0, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], 0, 0, P, page, heads, D, code, 0)
    _enqueue((_lib or load_library()).bv_pages_copy, dev, blob, pairs.data_ptr(), shape[0], upto)


# ---- prompts and rotary positions ----

_ROTARY = struct.Struct("@Qiifi")


def rotary_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, original: int = 0, low: float = 1.0, high: float = 32.0, device="cuda") -> torch.Tensor:
    """Frequencies for bv_cache_append_rotary, float64 [rot / 2]: base^(-2 i / rot), radians per position.

    ``factor`` > 1 stretches the context for which they were made: without ``original`` all of them are divided by it (positions interpolated
    linearly); with ``original``, the context's length before, by parts, as YaRN has it (Peng, Quesnelle, Fan, Shippole, 2023): those that turn fewer than
    ``low`` times in it are divided, those that turn more than ``high`` times are not, and between the two is a ramp that is linear in the index, from the last
    index with ``high`` turns or more to the first with ``low`` or fewer.  (The scale of queries and keys that goes with it is the caller's, ``mscale``.)"""
    if rot < 2 or rot % 2 or not base > 0 or not factor > 0:
        raise ValueError("rot must be even and at least 2, base and factor positive")
    f = torch.arange(rot // 2, dtype=torch.float64).mul_(-2.0 * math.log(base) / rot).exp_()
    if original <= 0 or factor == 1.0:
        return (f / factor).to(device)
    if not 0 < low < high:
        raise ValueError("low must be positive and below high")
    # (the index at which a pair turns `turns` times over the original context)
    at = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
    first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
    ramp = ((torch.arange(rot // 2, dtype=torch.float64) - first) / max(last - first, 0.001)).clamp_(0, 1)
    return (f * (1 - ramp) + f / factor * ramp).to(device)


def _offsets(offsets, B: int, dev: int):
    if B < 0 or offsets.dtype is not _I32 or offsets.dim() != 1 or not offsets.is_contiguous() or offsets.get_device() != dev:
        raise ValueError("offsets must be a contiguous int32 tensor [B + 1] on the same device")
    if offsets.shape[0] != B + 1:
        raise ValueError("offsets must be [B + 1]")
    return offsets.data_ptr()


def _packed(t, heads: int, D: int, dtype, dev: int, name: str):
    """(rows, heads, strides) of a tensor [tokens, heads, D] (heads = 0: any number)."""
    shape, st = t.shape, t.stride()
    if len(shape) != 3 or shape[2] != D or (heads and shape[1] != heads) or t.dtype is not dtype:
        raise ValueError("%s must be [tokens, heads, D] of one dtype" % name)
    if st[2] != 1 or t.get_device() != dev:
        raise ValueError("%s must have contiguous rows of D on one device" % name)
    return shape[0], shape[1], st


def bv_cache_append_rotary(q, k_new, v_new, k, v, table, lens, freq, n_new=None, offsets=None, interleaved: bool = False, mscale: float = 1.0, out_q=None,
                           out_k=None, stream=None):
    """Turns the queries and keys of the newest tokens by the angles of their positions and stores keys and values in their pages (see
    include/bv.h).

    ``q``, ``k_new``, ``v_new``: [B, n, heads, D], of which sequence b brings n (or n_new[b]), or with ``offsets`` (int32 [B + 1]) packed, [tokens, heads, D].
    ``q`` None: keys and values only.  ``freq`` float64 [rot / 2]: radians per position (``rotary_frequencies``); the first rot elements of a head turn,
    in pairs (i, i + rot / 2) or, ``interleaved``, (2 i, 2 i + 1), and are multiplied by ``mscale``.  ``out_q`` (may be ``q``) takes the queries, a tensor made
    here if None (rows that no sequence brings: zero in it); ``out_k`` (may be ``k_new``), if given, the keys.  Returns ``out_q``.  Autograd does not see it."""
    if stream is not None:
        return _on_stream(stream, lens, bv_cache_append_rotary, q, k_new, v_new, k, v, table, lens, freq, n_new, offsets, interleaved, mscale, out_q, out_k)
    if _fast is not None:
        r = _fast.rotary(q, k_new, v_new, k, v, table, lens, freq, n_new, offsets, interleaved, mscale, out_q, out_k)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    blob, B, heads, D, dtype, dev = _cache(k, v, table, lens)
    if freq.dtype is not torch.float64 or freq.dim() != 1 or not freq.is_contiguous() or freq.get_device() != dev or freq.shape[0] < 1:
        raise ValueError("freq must be a contiguous float64 tensor [rot / 2] on the cache's device")
    if offsets is not None and n_new is not None:
        raise ValueError("n_new goes with [B, n, heads, D], offsets with packed tokens")
    at = None if offsets is None else _offsets(offsets, B, dev)

    def rows(t, heads, name):
        if offsets is None:
            return _rows(t, B, heads, D, dtype, dev, name)
        n, heads, st = _packed(t, heads, D, dtype, dev, name)
        return n, heads, _STRIDES.pack(0, st[0], st[1])

    n, _, ks = rows(k_new, heads, "k_new")
    n_v, _, vs = rows(v_new, heads, "v_new")
    q_at, q_heads, qs, out_at, os_, k_at, ok = None, 0, None, None, None, None, None
    n_q = n
    if q is not None:
        n_q, q_heads, qs = rows(q, 0, "q")
        q_at = q.data_ptr()
        if out_q is None:
            out_q = q.new_empty(q.shape) if n_new is None and offsets is None else q.new_zeros(q.shape)
        else:
            _written(out_q, "out_q")
        n_o, _, os_ = rows(out_q, q_heads, "out_q")
        out_at = out_q.data_ptr()
        if n_o != n_q:
            raise ValueError("out_q must have the shape of q")
    elif out_q is not None:
        raise ValueError("out_q without q")
    if out_k is not None:
        _written(out_k, "out_k")
        n_o, _, ok = rows(out_k, heads, "out_k")
        k_at = out_k.data_ptr()
        if n_o != n:
            raise ValueError("out_k must have the shape of k_new")
    if n != n_v or n != n_q:
        raise ValueError("q, k_new and v_new must have one number of tokens")
    _written(k, "k")
    _written(v, "v")
    new = None if n_new is None else _counted(n_new, B, dev, "n_new")
    if B == 0 or (offsets is not None and n == 0):
        return out_q
    rotary = _ROTARY.pack(freq.data_ptr(), 2 * freq.shape[0], bool(interleaved), mscale, 0)
    _enqueue((_lib or load_library()).bv_cache_append_rotary, dev, blob, rotary, q_at, qs, q_heads, k_new.data_ptr(), ks, v_new.data_ptr(), vs, new, at, n, out_at, os_, k_at, ok)
    return out_q


def bv_prompt_attend(q, k, v, offsets, scale: Optional[float] = None, window: int = 0, sinks: int = 0, out=None, stream=None):
    """Causal attention of whole prompts that lie one after the other (see include/bv.h).

    ``q`` [tokens, q_heads, D], ``k``, ``v`` [tokens, heads, D] (float32 or bfloat16, any strides with contiguous rows); ``offsets`` int32 [B + 1]: sequence b is
    rows offsets[b] .. offsets[b + 1] - 1.  ``scale``: 1/sqrt(D) by default; ``window`` > 0: a token sees its last ``window`` tokens and the first
    ``sinks``.  Returns ``out`` [tokens, q_heads, D] (rows of no sequence are not written: zero in a tensor made here).  Forward only: what is returned has
    no autograd graph."""
    if stream is not None:
        return _on_stream(stream, offsets, bv_prompt_attend, q, k, v, offsets, scale, window, sinks, out)
    if _fast is not None:
        r = _fast.prompt(q, k, v, offsets, scale, window, sinks, out)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q must be [tokens, q_heads, D], k and v [tokens, heads, D]")
    D, dtype, dev = k.shape[2], k.dtype, k.get_device()
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError("queries, keys and values must be float32 or bfloat16, got %s" % dtype)
    if dev < 0:
        raise ValueError("expected CUDA tensors on one device")
    n, heads, ks = _packed(k, 0, D, dtype, dev, "k")
    n_v, _, vs = _packed(v, heads, D, dtype, dev, "v")
    n_q, q_heads, qs = _packed(q, 0, D, dtype, dev, "q")
    if n != n_v or n != n_q:
        raise ValueError("q, k and v must have one number of tokens")
    at = _offsets(offsets, offsets.shape[0] - 1 if offsets.dim() == 1 else -1, dev)
    if out is None:
        out = q.new_zeros((n, q_heads, D))
    else:
        _written(out, "out")
    n_o, _, os_ = _packed(out, q_heads, D, dtype, dev, "out")
    if n_o != n:
        raise ValueError("out must have the shape of q")
    if n == 0 or offsets.shape[0] == 1:
        return out
    pack = lambda st: _STRIDES.pack(st[0], st[1], 0)
    _enqueue((_lib or load_library()).bv_prompt_attend, dev, q.data_ptr(), pack(qs), k.data_ptr(), pack(ks), v.data_ptr(), pack(vs), at, offsets.shape[0] - 1, n, q_heads, heads, D,
             code, D ** -0.5 if scale is None else scale, window, sinks, out.data_ptr(), pack(os_))
    return out


# ---- rows of logits, cut ----

_CUT = struct.Struct("@4Qfiff")


def _cut(logits, temperature, top_k, top_p, min_p):
    """The packed settings: each a number, or a tensor with one for each row."""
    rows, dev = logits.shape[0], logits.get_device()

    def each(x, dtype, name):
        if not isinstance(x, torch.Tensor):
            return 0, x
        if x.dtype is not dtype or tuple(x.shape) != (rows,) or not x.is_contiguous() or x.get_device() != dev:
            raise ValueError("%s must be a number or a contiguous %s tensor [rows] on the logits' device" % (name, str(dtype)[6:]))
        return x.data_ptr(), 0

    t, k, p, m = each(temperature, torch.float32, "temperature"), each(top_k, _I32, "top_k"), each(top_p, torch.float32, "top_p"), each(min_p, torch.float32, "min_p")
    return _CUT.pack(t[0], k[0], p[0], m[0], t[1], min(max(k[1], 0), 2**31 - 1), p[1], m[1])


def _logits(t, name: str):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be [rows, V] with contiguous rows" % name)
    if not t.is_cuda:
        raise ValueError("expected CUDA tensors")
    return t.shape[0], t.shape[1]


def _cut_call(logits, uniforms, tokens, lse, out, temperature, top_k, top_p, min_p) -> None:
    rows, V = _logits(logits, "logits")
    code, dev = _dtype_code(logits), logits.get_device()
    if out is not None:
        if _logits(out, "the filtered logits") != (rows, V) or out.dtype is not logits.dtype or out.get_device() != dev:
            raise ValueError("the filtered logits must have the shape, dtype and device of the logits")
        if rows > 1 and out.stride(0) < V:
            raise ValueError("the filtered logits must not be an expanded tensor")
    cut = _cut(logits, temperature, top_k, top_p, min_p)
    if rows == 0:
        return
    ptr = lambda t: None if t is None else t.data_ptr()
    _enqueue((_lib or load_library()).bv_sample_filtered, dev, logits.data_ptr(), logits.stride(0), ptr(uniforms), rows, V, code, cut, ptr(tokens), ptr(lse), ptr(out),
             0 if out is None else out.stride(0))


def bv_sample_filtered(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, want_lse: bool = True, out_logits=None, stream=None):
    """The drafting step on cut rows (see include/bv.h): of ``logits`` [rows, V] (float32 or bfloat16, CUDA) the ``top_k`` largest (0: all), of these the smallest set
    with ``top_p`` of their mass, and of these what is at least ``min_p`` times as likely as the first; a token of each row drawn from that with ``uniforms``
    float32 [rows].  Each setting is a number or a tensor [rows] (float32; top_k int32).  Returns (tokens int32 [rows], lse float32 [rows] or None), lse of the kept
    tokens; ``out_logits`` (may be ``logits``), if given, takes the rows with all other logits at -inf."""
    if stream is not None:
        return _on_stream(stream, logits, bv_sample_filtered, logits, uniforms, temperature, top_k, top_p, min_p, want_lse, out_logits)
    if uniforms is None:
        raise ValueError("a token is drawn with uniforms; rows alone are bv_filter_logits'")
    if _fast is not None:
        r = _fast.sample(logits, uniforms, temperature, top_k, top_p, min_p, want_lse, out_logits)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    rows, _ = _logits(logits, "logits")
    if uniforms.shape != (rows,) or uniforms.dtype is not torch.float32 or not uniforms.is_contiguous() or uniforms.get_device() != logits.get_device():
        raise ValueError("uniforms must be a contiguous float32 tensor [rows] on the logits' device")
    tokens = torch.empty((rows,), dtype=torch.int32, device=logits.device)
    lse = torch.empty((rows,), dtype=torch.float32, device=logits.device) if want_lse else None
    _cut_call(logits, uniforms, tokens, lse, out_logits, temperature, top_k, top_p, min_p)
    return tokens, lse


def bv_filter_logits(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, stream=None):
    """``logits`` [rows, V] with all that bv_sample_filtered would not keep at -inf, in ``out`` (may be ``logits``; None: a new tensor)."""
    if stream is not None:
        return _on_stream(stream, logits, bv_filter_logits, logits, temperature, top_k, top_p, min_p, out)
    if out is None:
        out = torch.empty(tuple(logits.shape), dtype=logits.dtype, device=logits.device)
    if _fast is not None:
        r = _fast.sample(logits, None, temperature, top_k, top_p, min_p, False, out)
        if r is not NotImplemented:
            return r if r.__class__ is not int else _check(r)
    _cut_call(logits, None, None, None, out, temperature, top_k, top_p, min_p)
    return out
