"""Thin Python binding of libssq's C ABI (argument marshalling only).

Every step of the quantize / matmul path runs in the HIP kernels behind
``libssq.so``; this module only checks tensor dtypes and shapes, allocates
output tensors with torch and passes device pointers and the current stream.
It fails loudly if the library has not been built: there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Tuple

import torch

SIGNED_SYM, UNSIGNED_SYM, ASYM = 0, 1, 2
ASYM_MIN = 3    # min-max grid in the fp16-minimum layout (the ssq_*_min entry points)
MODES = {"signed_sym": SIGNED_SYM, "unsigned_sym": UNSIGNED_SYM, "asym": ASYM, "asym_min": ASYM_MIN}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libssq.so")

_EXPORTS = {
    "ssq_quantize": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                    ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_void_p]),
    "ssq_quantize_f32": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                        ctypes.c_void_p, ctypes.c_void_p]),
    "ssq_matmul": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                  ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]),
    "ssq_matmul_f32": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                      ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                      ctypes.c_void_p]),
    "ssq_matmul_workspace_size": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                                     ctypes.c_int, ctypes.c_int]),
    "ssq_matmul_ws": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                     ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_size_t, ctypes.c_void_p]),
    "ssq_strerror": (ctypes.c_char_p, [ctypes.c_int]),
}
_EXPORTS["ssq_matmul_noalloc"] = _EXPORTS["ssq_matmul"]
_Q_MIN = (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p])
_EXPORTS["ssq_quantize_min"] = _Q_MIN
_EXPORTS["ssq_quantize_min_f32"] = _Q_MIN
for _name in ("ssq_matmul_min", "ssq_matmul_min_f32", "ssq_matmul_min_ws"):
    _EXPORTS[_name] = (ctypes.c_int, list(_EXPORTS[_name.replace("_min", "")][1]))
_EXPORTS["ssq_sign_diagnostics"] = _Q_MIN
_EXPORTS["ssq_sign_diagnostics_f32"] = _Q_MIN
_EXPORTS["ssq_quantize_diag"] = (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                                ctypes.c_int] + [ctypes.c_void_p] * 4)
_EXPORTS["ssq_quantize_diag_f32"] = _EXPORTS["ssq_quantize_diag"]
_EXPORTS["ssq_quantize_act_q8"] = (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p])
_EXPORTS["ssq_matmul_q8"] = (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p] + _EXPORTS["ssq_matmul"][1][1:])
_EXPORTS["ssq_matmul_q8_min"] = _EXPORTS["ssq_matmul_q8"]
_EXPORTS["ssq_export_gguf"] = (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                              ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                              ctypes.c_void_p])
_EXPORTS["ssq_gguf_block_bytes"] = (ctypes.c_int64, [ctypes.c_int, ctypes.c_int])

_lib: Optional[ctypes.CDLL] = None


class SSQError(RuntimeError):
    """A libssq call returned a non-zero ssq_status."""

    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn}: {ssq_strerror(status)} (status {status})")
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libssq.so (once) and declare its signatures; raises if it is not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_08779_amd.build` (no fallback exists)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _EXPORTS.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def ssq_strerror(status: int) -> str:
    return lib().ssq_strerror(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    """Device address of a GPU tensor; a host tensor would hand a kernel a host pointer."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("ssq kernels take GPU tensors only (got a tensor on %s)" % t.device)
    return t.data_ptr()


# the current stream's handle without a Stream object around it (2 us less a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: torch.device) -> int:
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise SSQError(fn, status)


class _OnNullStream:
    """Orders a null-stream entry point (ssq_quantize*, the diagnostics) with the caller's
    current torch stream: the null stream waits for the work already queued on the
    current stream, and the current stream waits for the launch.  PyTorch's side streams
    are non-blocking, so without this a call inside ``torch.cuda.stream(s)`` could read
    W before s has written it, and s could read the outputs before they are written."""

    def __init__(self, device: torch.device):
        self.other = False
        if device.type == "cuda":        # a host tensor is refused by _ptr inside the block
            self.cur = torch.cuda.current_stream(device)
            self.null = torch.cuda.default_stream(device)
            self.other = self.cur.cuda_stream != self.null.cuda_stream

    def __enter__(self):
        if self.other:
            self.null.wait_stream(self.cur)
        return self

    def __exit__(self, *exc):
        if self.other:
            self.cur.wait_stream(self.null)
        return False


def ssq_quantize(W: torch.Tensor, group: int, q: int, mode: int,
                 out: Optional[Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]] = None):
    """Quantize W [rows, cols] (bf16 or fp32, on the GPU) group-wise.

    Returns (codes u8 [rows, cols*q/8], scales int16 [rows, cols/group] holding
    binary16 bit patterns, zp u8 [rows, cols/group] for ASYM, the binary16 minimums
    as int16 [rows, cols/group] for ASYM_MIN, else None).
    Runs on the null stream, like the C entry point, ordered after the work queued on
    the current stream and before the work queued on it afterwards.
    """
    if W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be a contiguous 2-D tensor")
    if W.dtype == torch.bfloat16:
        fn = "ssq_quantize"
    elif W.dtype == torch.float32:
        fn = "ssq_quantize_f32"
    else:
        raise TypeError("W must be bfloat16 or float32")
    rows, cols = W.shape
    if out is None:
        codes = torch.empty((rows, cols * q // 8), dtype=torch.uint8, device=W.device)
        scales = torch.empty((rows, cols // group if group else 0), dtype=torch.int16, device=W.device)
        meta_dtype = {ASYM: torch.uint8, ASYM_MIN: torch.int16}.get(mode)
        zp = (torch.empty((rows, cols // group if group else 0), dtype=meta_dtype, device=W.device)
              if meta_dtype is not None else None)
    else:
        codes, scales, zp = out
    with _OnNullStream(W.device):
        if mode == ASYM_MIN:
            fn = fn.replace("ssq_quantize", "ssq_quantize_min")
            st = getattr(lib(), fn)(_ptr(W), rows, cols, group, q, _ptr(codes), _ptr(scales), _ptr(zp))
        else:
            st = getattr(lib(), fn)(_ptr(W), rows, cols, group, q, mode, _ptr(codes), _ptr(scales), _ptr(zp))
    _check(fn, st)
    return codes, scales, zp


def ssq_matmul_workspace_size(M: int, N: int, K: int, group: int, q: int) -> int:
    """Bytes of workspace that let ssq_matmul_ws split the reduction (0: no benefit)."""
    return int(lib().ssq_matmul_workspace_size(M, N, K, group, q))


def ssq_matmul_workspace(M: int, N: int, K: int, group: int, q: int,
                         device=None) -> Optional[torch.Tensor]:
    """A zero-filled workspace tensor for ssq_matmul(..., workspace=...), or None."""
    n = ssq_matmul_workspace_size(M, N, K, group, q)
    return torch.zeros(n, dtype=torch.uint8, device=device or "cuda") if n else None


def ssq_matmul(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
               zp: Optional[torch.Tensor], N: int, K: int, group: int, q: int,
               out: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [M, N] = x [M, K] @ dequant(codes, scales, zp)^T on the current stream.

    x bf16 gives y bf16 (``ssq_matmul``, or ``ssq_matmul_ws`` when a workspace is
    given); x fp32 gives y fp32 (``ssq_matmul_f32``).  A ``zp`` of dtype int16
    holds binary16 minimums (the ASYM_MIN layout) and selects the ``*_min`` entry
    points; uint8 is the integer zero point; None the symmetric formats.
    """
    if x.dim() != 2 or not x.is_contiguous() or x.shape[1] != K:
        raise ValueError("x must be a contiguous [M, K] tensor")
    if x.dtype == torch.bfloat16:
        fn = "ssq_matmul"
    elif x.dtype == torch.float32:
        fn = "ssq_matmul_f32"
    else:
        raise TypeError("x must be bfloat16 or float32")
    if zp is not None and zp.dtype not in (torch.uint8, torch.int16):
        raise TypeError("zp must be uint8 zero points or int16 binary16 minimums")
    suffix = "_min" if zp is not None and zp.dtype == torch.int16 else ""
    M = x.shape[0]
    y = torch.empty((M, N), dtype=x.dtype, device=x.device) if out is None else out
    if workspace is not None and fn == "ssq_matmul":
        fn = "ssq_matmul" + suffix + "_ws"
        st = getattr(lib(), fn)(_ptr(x), M, _ptr(codes), _ptr(scales), _ptr(zp), N, K, group, q,
                                _ptr(y), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                _stream(x.device))
    else:
        fn = fn.replace("ssq_matmul", "ssq_matmul" + suffix)
        st = getattr(lib(), fn)(_ptr(x), M, _ptr(codes), _ptr(scales), _ptr(zp), N, K, group, q,
                                _ptr(y), _stream(x.device))
    _check(fn, st)
    return y


def ssq_matmul_noalloc(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                       zp: Optional[torch.Tensor], N: int, K: int, group: int, q: int,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """ssq_matmul for bf16 x whose split reduction uses the library's static scratch
    (``ssq_matmul_noalloc``) instead of a workspace; symmetric or u8 zero-point weights.
    With ``out`` given, the call allocates nothing."""
    if x.dim() != 2 or not x.is_contiguous() or x.shape[1] != K or x.dtype != torch.bfloat16:
        raise ValueError("x must be a contiguous bfloat16 [M, K] tensor")
    if zp is not None and zp.dtype != torch.uint8:
        raise TypeError("zp must be uint8 zero points or None")
    M = x.shape[0]
    y = torch.empty((M, N), dtype=x.dtype, device=x.device) if out is None else out
    st = lib().ssq_matmul_noalloc(_ptr(x), M, _ptr(codes), _ptr(scales), _ptr(zp), N, K, group, q,
                                  _ptr(y), _stream(x.device))
    _check("ssq_matmul_noalloc", st)
    return y


def ssq_sign_diagnostics(W: torch.Tensor, group: int, q: int, tally: bool = True, out=None):
    """Sec. 4 Remark 1 statistics of the signed absmax grid for every group of W.

    Returns (margin int16 [rows, cols/group] = |C_{-g*}| - |C_{g*}|, gain float32
    [rows, cols/group] = realised l2 gain of gamma* over -gamma*, tally int64 [3, 3]
    of groups by (sign margin, sign gain) or None).  `out` = (margin, gain, tally[9] or
    None) reuses buffers.  Runs on the null stream.
    """
    if W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be a contiguous 2-D tensor")
    if W.dtype == torch.bfloat16:
        fn = "ssq_sign_diagnostics"
    elif W.dtype == torch.float32:
        fn = "ssq_sign_diagnostics_f32"
    else:
        raise TypeError("W must be bfloat16 or float32")
    rows, cols = W.shape
    shape = (rows, cols // group if group else 0)
    if out is not None:
        margin, gain, t = out
        if (margin.dtype != torch.int16 or gain.dtype != torch.float32 or tuple(margin.shape) != shape
                or tuple(gain.shape) != shape or not (margin.is_contiguous() and gain.is_contiguous())
                or (t is not None and (t.dtype != torch.int64 or t.numel() != 9))):
            raise ValueError("out must be (int16 margin, float32 gain) of shape rows x cols/group "
                             "and an int64 tally of 9 elements or None")
    else:
        margin = torch.empty(shape, dtype=torch.int16, device=W.device)
        gain = torch.empty(shape, dtype=torch.float32, device=W.device)
        t = torch.empty(9, dtype=torch.int64, device=W.device) if tally else None
    with _OnNullStream(W.device):
        st = getattr(lib(), fn)(_ptr(W), rows, cols, group, q, _ptr(margin), _ptr(gain), _ptr(t))
    _check(fn, st)
    return margin, gain, (t.view(3, 3) if t is not None else None)


def ssq_quantize_act_q8(x: torch.Tensor, out=None):
    """Dynamic Q8_0 quantization of bf16 activations x [M, K] (App. C) on the current
    stream: returns (codes int8 [M, K], scales int16 [M, K/32] holding binary16 bits).
    ``out`` = (codes, scales) reuses buffers."""
    if x.dim() != 2 or not x.is_contiguous() or x.dtype != torch.bfloat16:
        raise ValueError("x must be a contiguous bfloat16 [M, K] tensor")
    M, K = x.shape
    if out is None:
        qx = torch.empty((M, K), dtype=torch.int8, device=x.device)
        dx = torch.empty((M, K // 32), dtype=torch.int16, device=x.device)
    else:
        qx, dx = out
    _check("ssq_quantize_act_q8", lib().ssq_quantize_act_q8(_ptr(x), M, K, _ptr(qx), _ptr(dx), _stream(x.device)))
    return qx, dx


def ssq_matmul_q8(qx: torch.Tensor, dx: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                  zp: Optional[torch.Tensor], N: int, K: int, group: int, q: int,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [M, N] bf16 from Q8_0 activations (``ssq_quantize_act_q8``) and packed weights
    by integer dot products (App. B.3), on the current stream.  ``zp``: None
    (symmetric), uint8 zero points, or int16 binary16 minimums (``ssq_matmul_q8_min``)."""
    if qx.dim() != 2 or not qx.is_contiguous() or qx.dtype != torch.int8 or qx.shape[1] != K:
        raise ValueError("qx must be a contiguous int8 [M, K] tensor")
    if zp is not None and zp.dtype not in (torch.uint8, torch.int16):
        raise TypeError("zp must be uint8 zero points or int16 binary16 minimums")
    fn = "ssq_matmul_q8_min" if zp is not None and zp.dtype == torch.int16 else "ssq_matmul_q8"
    M = qx.shape[0]
    y = torch.empty((M, N), dtype=torch.bfloat16, device=qx.device) if out is None else out
    st = getattr(lib(), fn)(_ptr(qx), _ptr(dx), M, _ptr(codes), _ptr(scales), _ptr(zp), N, K, group, q,
                            _ptr(y), _stream(qx.device))
    _check(fn, st)
    return y


def ssq_export_gguf(codes: torch.Tensor, scales: torch.Tensor, mins: Optional[torch.Tensor], rows: int,
                    cols: int, group: int, q: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The packed weights as GGUF blocks (uint8 [rows, cols/32, block bytes]: Q4_0/Q4_0s,
    Q4_1, Q2_0/Q2_0s or Q2_1 by q and whether ``mins`` is given), on the current stream."""
    if mins is not None and mins.dtype != torch.int16:
        raise TypeError("mins must be int16 binary16 minimums (ssq_quantize_min)")
    nbytes = int(lib().ssq_gguf_block_bytes(q, int(mins is not None)))
    if out is None:
        out = torch.empty((rows, cols // 32, max(nbytes, 1)), dtype=torch.uint8, device=codes.device)
    _check("ssq_export_gguf", lib().ssq_export_gguf(_ptr(codes), _ptr(scales), _ptr(mins), rows, cols, group, q,
                                                    _ptr(out), _stream(codes.device)))
    return out


def ssq_quantize_diag(W: torch.Tensor, group: int, q: int):
    """Signed-symmetric quantization fused with the sign-rule statistics (Sec. 4
    Remark 1): returns (codes, scales, margin int16, gain float32) in one pass over W,
    on the null stream."""
    if W.dim() != 2 or not W.is_contiguous():
        raise ValueError("W must be a contiguous 2-D tensor")
    if W.dtype == torch.bfloat16:
        fn = "ssq_quantize_diag"
    elif W.dtype == torch.float32:
        fn = "ssq_quantize_diag_f32"
    else:
        raise TypeError("W must be bfloat16 or float32")
    rows, cols = W.shape
    groups = cols // group if group else 0
    codes = torch.empty((rows, cols * q // 8), dtype=torch.uint8, device=W.device)
    scales = torch.empty((rows, groups), dtype=torch.int16, device=W.device)
    margin = torch.empty((rows, groups), dtype=torch.int16, device=W.device)
    gain = torch.empty((rows, groups), dtype=torch.float32, device=W.device)
    with _OnNullStream(W.device):
        st = getattr(lib(), fn)(_ptr(W), rows, cols, group, q, _ptr(codes), _ptr(scales), _ptr(margin), _ptr(gain))
    _check(fn, st)
    return codes, scales, margin, gain


# --- attention (include/ssq_attention.h) ------------------------------------------------------

_P, _I, _L, _F = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
_EXPORTS["ssq_page_tables"] = (_I, [_P, _P, _L, _P, _L, _P, _I, _P, _L, _L, _P, _P, _P, _P, _P, _P])
_EXPORTS["ssq_qk_norm_rope"] = (_I, [_P, _L, _P, _L, _P, _L, _L, _I, _I, _I, _P, _P, _F, _P, _P, _L, _P, _L, _P, _L,
                                     _P, _P, _P, _L, _I, _P])
_EXPORTS["ssq_attention_prompt"] = (_I, [_P, _L, _P, _L, _P, _L, _P, _L, _L, _I, _I, _I, _F, _P, _L, _P])
_EXPORTS["ssq_attention_decode"] = (_I, [_P, _L, _L, _I, _I, _I, _I, _F, _P, _P, _L, _I, _P, _L, _P, _L, _L, _P, _L, _P,
                                         ctypes.c_size_t, _P])
for _name in ("ssq_qk_norm_rope", "ssq_attention_prompt", "ssq_attention_decode"):
    _EXPORTS[_name + "_f32"] = _EXPORTS[_name]
_EXPORTS["ssq_attention_decode_workspace_size"] = (ctypes.c_size_t, [_L, _I, _I, _I, _I, _L, _L])


_entries: dict = {}
_PACKED = torch.contiguous_format       # of outputs, whatever their inputs' strides (empty_like takes half of empty's time)


def _entry(name: str, dtype: torch.dtype):
    """The C function for tensors of dtype, and its name."""
    found = _entries.get((name, dtype))
    if found is None:
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("tensors must be bfloat16 or float32")
        full = name if dtype == torch.bfloat16 else name + "_f32"
        found = _entries[name, dtype] = (getattr(lib(), full), full)
    return found


def _heads(t: torch.Tensor, what: str, dtype: torch.dtype, tokens: Optional[int] = None) -> int:
    """Elements between the rows of t [tokens, heads, head_dim], whose rows are contiguous."""
    if t.dim() != 3 or t.dtype != dtype:
        raise ValueError(f"{what} must be a [tokens, heads, head_dim] tensor of {dtype}")
    n, heads, dim = t.shape
    if tokens is not None and n != tokens:
        raise ValueError(f"{what} has {n} tokens, not {tokens}")
    rows, between, one = t.stride()
    if one != 1 or (between != dim and heads > 1):
        raise ValueError(f"the heads of a token of {what} must be contiguous")
    return rows if n > 1 else heads * dim


def _flat(t: torch.Tensor, what: str, dtype: torch.dtype, shape: Tuple[int, ...]) -> int:
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    if not t.is_cuda:
        raise ValueError("ssq kernels take GPU tensors only (got a tensor on %s)" % t.device)
    return t.data_ptr()


def ssq_page_tables(held: torch.Tensor, added: torch.Tensor, free_pages: torch.Tensor, table: torch.Tensor,
                    page_size: int, tokens: int, taken: Optional[torch.Tensor] = None, out=None):
    """Page table, slots and positions of a step's new tokens on the current stream.

    Request r holds ``held[r]`` tokens and adds ``added[r]`` (int32); pages it needs come from
    ``free_pages`` (int32), request after request, from entry ``taken`` (int32 [1]; None: 0) on.
    ``table`` (int32 [requests, pages]) is updated in place.  Returns (starts [requests + 1],
    lens [requests], positions [tokens], slots [tokens], taken after [1], table), all int32;
    ``tokens`` may exceed the sum of ``added`` (padding: position 0, slot -1).  ``out`` = the
    first five reuses buffers, which must not be those of another argument (``held`` for lens)."""
    if held.dim() != 1 or table.dim() != 2:
        raise ValueError("held must be [requests] and table [requests, pages]")
    n, width = table.shape
    i32, dev, one = torch.int32, held.device, (n,)
    if out is None:
        if tokens < 0:
            raise ValueError("tokens must not be negative")
        # one allocation, cut up
        buf = torch.empty(2 * n + 2 * tokens + 2, dtype=i32, device=dev)
        starts, lens, positions, slots, after = torch.split_with_sizes(buf, (n + 1, n, tokens, tokens, 1))
        at = _ptr(buf)
        to = at, at + 4 * (n + 1), at + 4 * (2 * n + 1), at + 4 * (2 * n + 1 + tokens), at + 4 * (2 * n + 1 + 2 * tokens)
    else:
        starts, lens, positions, slots, after = out
        to = (_flat(starts, "starts", i32, (n + 1,)), _flat(lens, "lens", i32, one), _flat(positions, "positions", i32, (tokens,)),
              _flat(slots, "slots", i32, (tokens,)), _flat(after, "taken after", i32, (1,)))
    fn, name = _entry("ssq_page_tables", torch.bfloat16)
    st = fn(_flat(held, "held", i32, one), _flat(added, "added", i32, one), n,
            _flat(free_pages, "free_pages", i32, free_pages.shape[:1]), free_pages.numel(),
            None if taken is None else _flat(taken, "taken", i32, (1,)), page_size, _flat(table, "table", i32, (n, width)),
            width, tokens, *to, _stream(dev))
    if st:
        _check(name, st)
    return starts, lens, positions, slots, after, table


def ssq_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, rope: torch.Tensor,
                     q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     v: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                     k_pages: Optional[torch.Tensor] = None, v_pages: Optional[torch.Tensor] = None, out=None):
    """Norms (where a gain is given) and position rotation of q [tokens, q_heads, head_dim] and
    k [tokens, kv_heads, head_dim], on the current stream; returns (q, k) rotated.

    bf16 (or fp32: ``ssq_qk_norm_rope_f32``); tokens may be strided, as in the rows of one fused
    projection.  ``rope`` fp32 [rows, head_dim] holds cosines, then sines, of each position.
    With ``slots`` (int32 [tokens], ``ssq_page_tables``) the rotated k and the given v also go to
    the caches k_pages, v_pages [pages, kv_heads, page_size, head_dim].  ``out`` = (q, k) reuses
    buffers (k may be None with a cache; they may be q and k themselves)."""
    dtype = q.dtype
    fn, name = _entry("ssq_qk_norm_rope", dtype)
    qs, ks = _heads(q, "q", dtype), _heads(k, "k", dtype, q.shape[0])
    tokens, hq, dim = q.shape
    hk = k.shape[1]
    if k.shape[2] != dim or rope.dim() != 2 or rope.shape[1] != dim:
        raise ValueError("q, k and rope must have the same head_dim")
    cache = slots is not None
    if cache != (k_pages is not None) or cache != (v_pages is not None) or (cache and v is None):
        raise ValueError("slots, k_pages and v_pages go together, with v")
    vs = pages = page_size = 0
    vp = sp = kp = pp = None
    if cache:
        vs, vp = _heads(v, "v", dtype, tokens), _ptr(v)
        if v.shape != k.shape or k_pages.dim() != 4:
            raise ValueError("v must be like k, and the caches [pages, kv_heads, page_size, head_dim]")
        pages, _, page_size, _ = shape = k_pages.shape
        if shape[1] != hk or shape[3] != dim:
            raise ValueError("the caches must be [pages, kv_heads, page_size, head_dim] of k's heads")
        kp, pp = _flat(k_pages, "k_pages", dtype, shape), _flat(v_pages, "v_pages", dtype, shape)
        sp = _flat(slots, "slots", torch.int32, (tokens,))
    if out is None:
        qos, kos = hq * dim, hk * dim
        q_out, k_out = torch.empty_like(q, memory_format=_PACKED), torch.empty_like(k, memory_format=_PACKED)
    else:
        q_out, k_out = out
        if q_out.shape != q.shape or (k_out is not None and k_out.shape != k.shape):
            raise ValueError("out must be tensors like q and k")
        qos = _heads(q_out, "q_out", dtype)
        kos = 0 if k_out is None else _heads(k_out, "k_out", dtype)
    st = fn(_ptr(q), qs, _ptr(k), ks, vp, vs, tokens, hq, hk, dim,
            None if q_gain is None else _flat(q_gain, "q_gain", dtype, (dim,)),
            None if k_gain is None else _flat(k_gain, "k_gain", dtype, (dim,)), eps,
            _flat(positions, "positions", torch.int32, (tokens,)), _flat(rope, "rope", torch.float32, (rope.shape[0], dim)),
            rope.shape[0], _ptr(q_out), qos, _ptr(k_out), kos, sp, kp, pp, pages, page_size, _stream(q.device))
    if st:
        _check(name, st)
    return q_out, k_out


def ssq_attention_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor,
                         scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal attention of packed prompts on the current stream: q [tokens, q_heads, head_dim],
    k and v [tokens, kv_heads, head_dim], bf16 or fp32, tokens may be strided.  ``starts`` (int32
    [requests + 1]) holds the first token of each sequence and the end of the last; tokens behind
    it give zeros.  ``scale`` defaults to 1 / sqrt(head_dim)."""
    dtype = q.dtype
    fn, name = _entry("ssq_attention_prompt", dtype)
    qs, ks = _heads(q, "q", dtype), _heads(k, "k", dtype, q.shape[0])
    vs = _heads(v, "v", dtype, q.shape[0])
    tokens, hq, dim = q.shape
    hk = k.shape[1]
    if k.shape != v.shape or k.shape[2] != dim:
        raise ValueError("k and v must have the same shape, and q's head_dim")
    if starts.dim() != 1 or starts.shape[0] < 1:
        raise ValueError("starts must hold requests + 1 values")
    if out is None:
        out, os_ = torch.empty_like(q, memory_format=_PACKED), hq * dim
    elif out.shape != q.shape:
        raise ValueError("out must be a tensor like q")
    else:
        os_ = _heads(out, "out", dtype)
    st = fn(_ptr(q), qs, _ptr(k), ks, _ptr(v), vs, _flat(starts, "starts", torch.int32, starts.shape), starts.shape[0] - 1,
            tokens, hq, hk, dim, dim ** -0.5 if scale is None else scale, _ptr(out), os_, _stream(q.device))
    if st:
        _check(name, st)
    return out


def ssq_attention_decode_workspace_size(requests: int, fresh: int, q_heads: int, kv_heads: int, head_dim: int,
                                        max_len: int, prefix: int = 0) -> int:
    """Bytes of scratch that let ssq_attention_decode split long caches and share a prefix."""
    return int(lib().ssq_attention_decode_workspace_size(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix))


def _fresh_rows(q: torch.Tensor) -> int:
    """Elements between the tokens of q [requests, fresh, q_heads, head_dim]."""
    if q.dim() != 4 or q.stride(3) != 1 or (q.stride(2) != q.shape[3] and q.shape[2] > 1) or (
            q.shape[0] > 1 and q.shape[1] > 1 and q.stride(0) != q.shape[1] * q.stride(1)):
        raise ValueError("q must be [requests, fresh, q_heads, head_dim], its tokens equally far apart and each contiguous")
    return q.stride(1) if q.shape[1] > 1 else q.stride(0) if q.shape[0] > 1 else q.shape[2] * q.shape[3]


def ssq_attention_decode(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor,
                         lens: torch.Tensor, max_len: int, prefix: int = 0, scale: Optional[float] = None,
                         out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the new tokens q [requests, fresh, q_heads, head_dim] over the paged caches
    [pages, kv_heads, page_size, head_dim], bf16 or fp32, on the current stream.

    Request r has ``lens[r]`` tokens in the cache (int32, at most ``max_len``), its ``fresh`` new
    ones the last of them, in the pages of ``table[r]`` (int32 [requests, pages]); the first
    ``prefix`` tokens are the same for all requests and are read from request 0's pages, once.
    ``workspace`` (uint8, any contents, ``ssq_attention_decode_workspace_size`` bytes) is allocated
    where it is not given; ``scale`` defaults to 1 / sqrt(head_dim)."""
    dtype = q.dtype
    fn, name = _entry("ssq_attention_decode", dtype)
    stride = _fresh_rows(q)
    n, fresh, hq, dim = q.shape
    if k_pages.dim() != 4 or k_pages.shape[3] != dim:
        raise ValueError("the caches must be [pages, kv_heads, page_size, head_dim]")
    pages, hk, page_size, _ = k_pages.shape
    if table.dim() != 2:
        raise ValueError("table must be a contiguous int32 [requests, pages] tensor")
    width = table.shape[1]
    if out is None:
        out = torch.empty_like(q, memory_format=_PACKED)
    elif out.shape != q.shape or out.dtype != dtype or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor like q")
    if workspace is None:
        size = lib().ssq_attention_decode_workspace_size(n, fresh, hq, hk, dim, max_len, prefix)
        if size:
            workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    elif not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    shape = k_pages.shape
    st = fn(_ptr(q), stride, n, fresh, hq, hk, dim, dim ** -0.5 if scale is None else scale, _flat(k_pages, "k_pages", dtype, shape),
            _flat(v_pages, "v_pages", dtype, shape), pages, page_size, _flat(table, "table", torch.int32, (n, width)), width,
            _flat(lens, "lens", torch.int32, (n,)), max_len, prefix, _ptr(out), hq * dim, _ptr(workspace),
            0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(q.device))
    if st:
        _check(name, st)
    return out


# --- the paged cache in 4 bits, and pages of any cache (include/ssq_cache.h) -------------------

for _name, _args in (("ssq_kv4_store", [_P, _L, _P, _L, _L, _I, _I, _P, _P, _L, _I, _P, _L, _P, _L, _P]),
                     ("ssq_attention_decode_kv4", [_P, _L, _L, _I, _I, _I, _I, _F, _P, _L, _I, _P, _L, _P, _L, _L, _P, _L, _P,
                                                   ctypes.c_size_t, _P])):
    _EXPORTS[_name] = _EXPORTS[_name + "_f32"] = (_I, _args)
_EXPORTS["ssq_attention_decode_kv4_workspace_size"] = _EXPORTS["ssq_attention_decode_workspace_size"]
_EXPORTS["ssq_page_fork"] = (_I, [_P, _L, _P, _P, _L, _L, _P, _L, _P, _I, _P, _L, _P, _P, _P, _P, _P])
_EXPORTS["ssq_page_collect"] = (_I, [_P, _L, _P, _L, _I, _L, _P, _P, _P, _P, ctypes.c_size_t, _P])
_EXPORTS["ssq_page_compact"] = (_I, [_P, _L, _P, _L, _I, _L, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P])
_EXPORTS["ssq_page_collect_workspace_size"] = (ctypes.c_size_t, [_L, _I])
_EXPORTS["ssq_page_copy"] = (_I, [_P, _I, _L, _L, _P, _P, _L, _P])


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(fn, name: str, first: torch.Tensor, others, *args) -> None:
    """fn(*args, stream) on the current stream of the device of ``first``, where all ``others`` (or None) have to be."""
    index = first.get_device()
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"all tensors must be on one device (got {first.device} and {t.device})")
    if index == _current_device():
        st = fn(*args, _stream(first.device))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _stream(first.device))
    if st:
        _check(name, st)


def ssq_kv4_cache(pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda") -> torch.Tensor:
    """An empty cache in 4 bits, of both keys and values: uint8 [pages, kv_heads, 2,
    page_size * 9 * head_dim // 16] (the layout is in include/ssq_cache.h)."""
    return torch.zeros((pages, kv_heads, 2, page_size * 9 * head_dim // 16), dtype=torch.uint8, device=device)


def _kv4(cache: torch.Tensor, heads: int, dim: int) -> Tuple[int, int, int]:
    """Pointer, pages and page size of a 4-bit cache."""
    if cache.dim() != 4 or cache.shape[1] != heads or cache.shape[2] != 2 or cache.shape[3] * 16 % (9 * dim or 1):
        raise ValueError("the cache must be [pages, kv_heads, 2, page_size * 9 * head_dim // 16] of these heads")
    return _flat(cache, "cache", torch.uint8, cache.shape), cache.shape[0], cache.shape[3] * 16 // (9 * dim or 1)


def ssq_kv4_store(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: torch.Tensor, held=None):
    """Keys and values [tokens, kv_heads, head_dim] (bf16 or fp32; tokens may be strided) onto the signed
    absmax grid in 4 bits and into their ``slots`` (int32 [tokens]) of ``cache`` (``ssq_kv4_cache``), on the
    current stream.  With ``held=True`` the rows as the cache holds them are returned, (k, v), for a
    prompt's own attention; ``held`` = (k, v) writes them to those tensors, which may be k and v."""
    dtype = k.dtype
    fn, name = _entry("ssq_kv4_store", dtype)
    ks, vs = _heads(k, "k", dtype), _heads(v, "v", dtype, k.shape[0])
    tokens, hk, dim = k.shape
    if v.shape != k.shape:
        raise ValueError("v must be like k")
    cp, pages, page_size = _kv4(cache, hk, dim)
    khs = vhs = 0
    khp = vhp = None
    if held is True:
        held = torch.empty_like(k, memory_format=_PACKED), torch.empty_like(v, memory_format=_PACKED)
        khs = vhs = hk * dim
        khp, vhp = held[0].data_ptr(), held[1].data_ptr()
    elif held:
        if held[0].shape != k.shape or held[1].shape != v.shape:
            raise ValueError("held must be tensors like k and v")
        khs, vhs = _heads(held[0], "held k", dtype), _heads(held[1], "held v", dtype)
        khp, vhp = _ptr(held[0]), _ptr(held[1])
    _launch(fn, name, k, (v, slots, cache, *(held or ())), _ptr(k), ks, _ptr(v), vs, tokens, hk, dim,
            _flat(slots, "slots", torch.int32, (tokens,)), cp, pages, page_size, khp, khs, vhp, vhs)
    return held or None


@functools.lru_cache(maxsize=256)
def _decode_kv4_bytes(*sizes: int) -> int:
    return int(lib().ssq_attention_decode_kv4_workspace_size(*sizes))


def ssq_attention_decode_kv4_workspace_size(requests: int, fresh: int, q_heads: int, kv_heads: int, head_dim: int,
                                            max_len: int, prefix: int = 0) -> int:
    """Bytes of scratch that let ssq_attention_decode_kv4 split long caches and share a prefix."""
    return _decode_kv4_bytes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix)


def ssq_attention_decode_kv4(q: torch.Tensor, cache: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, max_len: int,
                             prefix: int = 0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                             workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``ssq_attention_decode`` over a cache in 4 bits (``ssq_kv4_cache``): the same arguments, with one
    ``cache`` in place of the two.  ``workspace`` (uint8, any contents,
    ``ssq_attention_decode_kv4_workspace_size`` bytes) is allocated where it is not given."""
    dtype = q.dtype
    fn, name = _entry("ssq_attention_decode_kv4", dtype)
    stride = _fresh_rows(q)
    n, fresh, hq, dim = q.shape
    if cache.dim() != 4 or table.dim() != 2:
        raise ValueError("the cache must be [pages, kv_heads, 2, bytes] and table [requests, pages]")
    hk, width = cache.shape[1], table.shape[1]
    cp, pages, page_size = _kv4(cache, hk, dim)
    if out is None:
        out = torch.empty_like(q, memory_format=_PACKED)
    elif out.shape != q.shape or out.dtype != dtype or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor like q")
    if workspace is None:
        size = _decode_kv4_bytes(n, fresh, hq, hk, dim, max_len, prefix)
        if size:
            workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    elif not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _launch(fn, name, q, (cache, table, lens, out, workspace), _ptr(q), stride, n, fresh, hq, hk, dim,
            dim ** -0.5 if scale is None else scale, cp, pages, page_size, _flat(table, "table", torch.int32, (n, width)), width,
            _flat(lens, "lens", torch.int32, (n,)), max_len, prefix, _ptr(out), hq * dim, _ptr(workspace),
            0 if workspace is None else workspace.numel() * workspace.element_size())
    return out


def ssq_page_fork(parents: torch.Tensor, lens: torch.Tensor, table: torch.Tensor, free_pages: torch.Tensor, page_size: int,
                  taken: Optional[torch.Tensor] = None, width: Optional[int] = None, out=None):
    """Tables of requests that continue others, on the current stream: request i has the pages of row
    ``parents[i]`` (int32; outside the rows: none) of ``table`` (int32 [rows, pages], ``lens`` [rows]
    tokens), but a new page from ``free_pages`` (entry ``taken`` on) in place of a last page that is not full and
    that an earlier request continues.  Returns (table [requests, width], lens, src, dst [requests], taken after [1]),
    int32; ``width`` defaults to that of ``table``.  The pages src -> dst (-1: none) are to be copied in
    every layer (``ssq_page_copy``).  ``out`` = these five reuses buffers, which must not be those of another argument."""
    if parents.dim() != 1 or table.dim() != 2:
        raise ValueError("parents must be [requests] and table [rows, pages]")
    i32, dev, n = torch.int32, parents.device, parents.shape[0]
    rows, stride = table.shape
    if out is None:
        width = stride if width is None else width
        if width < 0:
            raise ValueError("width must not be negative")
        # one allocation, cut up
        buf = torch.empty(n * width + 3 * n + 1, dtype=i32, device=dev)
        table_out, lens_out, src, dst, after = torch.split_with_sizes(buf, (n * width, n, n, n, 1))
        table_out = table_out.view(n, width)
        at = _ptr(buf)
        to = at, at + 4 * n * width, at + 4 * n * (width + 1), at + 4 * n * (width + 2), at + 4 * n * (width + 3)
    else:
        table_out, lens_out, src, dst, after = out
        if table_out.dim() != 2 or (width is not None and table_out.shape[1] != width):
            raise ValueError("out's table must be [requests, width]")
        width = table_out.shape[1]
        to = (_flat(table_out, "table out", i32, (n, width)), _flat(lens_out, "lens out", i32, (n,)), _flat(src, "src", i32, (n,)),
              _flat(dst, "dst", i32, (n,)), _flat(after, "taken after", i32, (1,)))
    fn, name = _entry("ssq_page_fork", torch.bfloat16)
    _launch(fn, name, parents, (lens, table, free_pages, taken, table_out, lens_out, src, dst, after), _flat(parents, "parents", i32, (n,)), n,
            _flat(lens, "lens", i32, (rows,)), _flat(table, "table", i32, (rows, stride)), rows, stride,
            _flat(free_pages, "free_pages", i32, free_pages.shape[:1]), free_pages.numel(),
            None if taken is None else _flat(taken, "taken", i32, (1,)), page_size, to[0], width, *to[1:])
    return table_out, lens_out, src, dst, after


@functools.lru_cache(maxsize=64)
def _collect_bytes(pages: int, compact: bool) -> int:
    return int(lib().ssq_page_collect_workspace_size(pages, int(compact)))


# Bytes of a workspace that lies behind the outputs, in their allocation (1.4 us less of the host than one of its own, of 9 in all
# for 9000 pages).  A larger one (a compaction of 116000 pages) is freed with the call, not kept by whoever keeps an output.
_SCRATCH_INSIDE = 1 << 20


def _collect(name: str, lens, table, page_size, pages, pinned, sizes, out, workspace, compact: bool):
    """ssq_page_collect or ssq_page_compact into int32 arrays of `sizes`, allocated with the workspace where they are not given."""
    if lens.dim() != 1 or table.dim() != 2:
        raise ValueError("lens must be [requests] and table [requests, pages]")
    if pages < 0:
        raise ValueError("pages must not be negative")
    n, width = table.shape
    i32, need = torch.int32, _collect_bytes(pages, compact)
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if out is None:
        total = sum(sizes)
        inside = workspace is None and need <= _SCRATCH_INSIDE
        scratch = -total % 64 + (need + 3) // 4 if inside else 0
        buf = torch.empty(total + scratch, dtype=i32, device=lens.device)
        base = _ptr(buf)
        out = torch.split_with_sizes(buf, (*sizes, scratch))[:-1]
        to, at = [], base
        for size in sizes:
            to.append(at)
            at += 4 * size
        if compact:
            out = (out[0].view(n, width), *out[1:])
        if inside:                              # from the next 256 bytes on
            scratch_at, scratch_bytes = base + 4 * (total + -total % 64), need
        elif workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=lens.device)
    else:
        to = [_flat(x, "an output", i32, (n, width) if compact and i == 0 else (size,)) for i, (x, size) in enumerate(zip(out, sizes))]
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=lens.device)
    if workspace is not None:
        scratch_at, scratch_bytes = _ptr(workspace), workspace.numel() * workspace.element_size()
    fn, name = _entry(name, torch.bfloat16)
    _launch(fn, name, lens, (table, pinned, *out, workspace), _flat(lens, "lens", i32, (n,)), n, _flat(table, "table", i32, (n, width)), width, page_size,
            pages, None if pinned is None else _flat(pinned, "pinned", torch.uint8, (pages,)), *to, scratch_at, scratch_bytes)
    return out


def ssq_page_collect(lens: torch.Tensor, table: torch.Tensor, page_size: int, pages: int, pinned: Optional[torch.Tensor] = None,
                     out=None, workspace: Optional[torch.Tensor] = None):
    """The pages of a pool of ``pages`` that no request holds, on the current stream: request r holds the
    first ceil(lens[r] / page_size) entries of ``table[r]`` (int32 [requests, pages]); ``pinned`` (uint8 [pages])
    is not 0 for pages that are held in any case.  Returns (free_pages [pages], ascending, then -1; count [1]), int32,
    in one allocation.
    ``out`` = these two reuses buffers; ``workspace`` (uint8, any contents, ``ssq_page_collect_workspace_size`` bytes)
    is allocated where it is not given."""
    return _collect("ssq_page_collect", lens, table, page_size, pages, pinned, (pages, 1), out, workspace, False)


def ssq_page_compact(lens: torch.Tensor, table: torch.Tensor, page_size: int, pages: int, pinned: Optional[torch.Tensor] = None,
                     out=None, workspace: Optional[torch.Tensor] = None):
    """``ssq_page_collect`` with the held pages brought to the front of the pool: returns (table with the new
    numbers, free_pages [pages] and count [1] after the moves, src, dst [pages // 2]: the moves, then -1, moved [1]), int32.
    The moves are to be made in every layer (``ssq_page_copy``) before its cache is next used.  ``out`` = these
    six reuses buffers; its table may be ``table`` itself."""
    return _collect("ssq_page_compact", lens, table, page_size, pages, pinned, (table.numel(), pages, 1, pages // 2, pages // 2, 1), out, workspace, True)


def ssq_page_collect_workspace_size(pages: int, compact: bool = False) -> int:
    """Bytes of scratch for ssq_page_collect, or (``compact``) for ssq_page_compact."""
    return _collect_bytes(pages, bool(compact))


def ssq_page_copy(caches, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Page ``src[i]`` of every cache into its page ``dst[i]`` (int32; negative: nothing), on the current stream.
    ``caches``: contiguous tensors [pages, ...] of one device whose pages have the same number of bytes, such as
    all layers' k_pages and v_pages, or their 4-bit caches; they must not overlap.  No page may be named twice in dst,
    or in both."""
    caches = list(caches)
    if not caches:
        return
    shape, dtype, size = caches[0].shape, caches[0].dtype, caches[0].element_size()
    if not shape or src.dim() != 1:
        raise ValueError("caches must be [pages, ...], src and dst [entries]")
    pages, page_bytes = shape[0], shape[1:].numel() * size
    for c in caches:
        alike = c.shape == shape and c.dtype == dtype or c.dim() > 0 and c.shape[0] == pages and c.shape[1:].numel() * c.element_size() == page_bytes
        if not alike or not c.is_contiguous():
            raise ValueError("caches must be contiguous, on one device, and have the same pages and bytes a page")
    fn, name = _entry("ssq_page_copy", torch.bfloat16)
    _launch(fn, name, caches[0], (*caches[1:], src, dst), (ctypes.c_void_p * len(caches))(*(_ptr(c) for c in caches)), len(caches), page_bytes, pages,
            _flat(src, "src", torch.int32, src.shape), _flat(dst, "dst", torch.int32, src.shape), src.shape[0])
