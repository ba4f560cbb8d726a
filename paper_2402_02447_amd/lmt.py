"""The operators at the two ends of a language model's training step in libbca.so (include/lmt.h): embedding lookup and
its table's gradient, 8-bit quantisation and products, cross entropy with its gradient.

Same names as the C ABI without the prefix.  Arguments are torch tensors on the current device, whose shapes, strides and types
give the rest; outputs are tensors that the caller has allocated.  Calls only enqueue on `stream` (a
``torch.cuda.Stream``, an integer handle, or None for the default stream, not for torch's current one), and write through the tensors'
addresses: autograd sees neither the call nor, in its version counters, what it has changed.  What does not fit together raises ValueError,
what the library refuses LmtError.  There is no CPU fallback: without the built library or the extension module
_calls every call raises."""
from __future__ import annotations

import ctypes as C

from .binding import load_library

LMT_F32, LMT_F16, LMT_BF16, LMT_E4M3, LMT_E5M2, LMT_I32, LMT_I64 = range(7)
LMT_STATUS_BAD_TOKEN, LMT_STATUS_BAD_TARGET = 1, 2
LMT_ACCUMULATE, LMT_TILE_SCALES, LMT_FP32_SUMS = 1, 2, 4
LMT_MAX_ROWS, LMT_MAX_WIDTH = 0x7FFFFF00, 0x7FFFFF
_ERR = {-1: "LMT_ERR_NULL", -2: "LMT_ERR_ARG", -3: "LMT_ERR_LIMIT", -4: "LMT_ERR_HIP", -5: "LMT_ERR_ALIGN", -6: "LMT_ERR_WORKSPACE"}
_BYTES = 7                          # uint8: scales and workspaces

EXPORTS = ["lmt_embed", "lmt_embed_grad", "lmt_embed_grad_workspace", "lmt_fp8_row_bytes", "lmt_scale_row_bytes",
           "lmt_quantize", "lmt_matmul_workspace", "lmt_matmul", "lmt_cross_entropy", "lmt_last_error"]


class LmtError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_ERR.get(code, code)}: {msg}")
        self.code = code


_library = _calls = _table = None


def _lib():
    """The library with this header's functions declared."""
    global _library
    if _library is None:
        L = load_library()
        vp, i32, i64, u32, u64, dbl = C.c_void_p, C.c_int, C.c_int64, C.c_uint32, C.c_uint64, C.c_double
        L.lmt_embed.argtypes = [vp, i32, u64, u64, u64, vp, i32, u64, dbl, vp, i32, u64, vp, vp]
        L.lmt_embed_grad.argtypes = [vp, i32, u64, vp, i32, u64, dbl, i64, vp, i32, u64, u64, u64, u32, vp, vp, u64, vp]
        L.lmt_quantize.argtypes = [vp, i32, u64, u64, u64, i32, u32, vp, vp, vp, vp, vp]
        L.lmt_matmul.argtypes = [vp, i32, vp, vp, i32, vp, u64, u64, u64, vp, i32, u64, u32, vp, u64, vp]
        L.lmt_cross_entropy.argtypes = [vp, i32, u64, u64, u64, vp, i32, i64, vp, vp, vp, vp, u64, vp, vp]
        for name in ("lmt_embed_grad_workspace", "lmt_matmul_workspace"):
            getattr(L, name).argtypes, getattr(L, name).restype = [u64, u64, u64], u64
        for name in ("lmt_fp8_row_bytes", "lmt_scale_row_bytes"):
            getattr(L, name).argtypes, getattr(L, name).restype = [u64], u64
        L.lmt_last_error.restype = C.c_char_p
        for name in EXPORTS:
            getattr(L, name)
        _library = L
    return _library


def _connect():
    """The extension module and its table of this library's functions."""
    global _calls, _table
    L = _lib()
    import torch
    try:
        from . import _calls as module
    except ImportError as e:
        raise ImportError("the extension module _calls has not been built (python -c 'import __graft_entry__ as g; g.build()')") from e
    types = {torch.float32: LMT_F32, torch.float16: LMT_F16, torch.bfloat16: LMT_BF16, torch.float8_e4m3fn: LMT_E4M3,
             torch.float8_e5m2: LMT_E5M2, torch.int32: LMT_I32, torch.int64: LMT_I64, torch.uint8: _BYTES}
    addresses = [C.cast(getattr(L, f), C.c_void_p).value for f in ("lmt_embed", "lmt_embed_grad", "lmt_quantize", "lmt_matmul", "lmt_cross_entropy")]
    _calls, _table = module, module.lmt_connect(*addresses, types, torch.cuda.current_device)


def _check(rc: int) -> None:
    if rc != 0:
        raise LmtError(rc, _lib().lmt_last_error().decode())


def embed(table, tokens, out, scale: float = 1.0, status=None, stream=None) -> None:
    """out[t] = scale * table[tokens[t]].  table: [vocab, width]; tokens: [n] int32 or int64; out: [n, width]; status: int32
    or None (LMT_STATUS_BAD_TOKEN)."""
    if _table is None:
        _connect()
    _check(_calls.lmt_embed(_table, table, tokens, out, scale, status, stream))


def embed_grad_workspace(n_tokens: int, vocab: int, width: int) -> int:
    """Bytes of the uint8 tensor that embed_grad works in."""
    return int(_lib().lmt_embed_grad_workspace(n_tokens, vocab, width))


def embed_grad(grad_out, tokens, grad, workspace, scale: float = 1.0, skip_token: int = -1, accumulate: bool = False,
               status=None, stream=None) -> None:
    """grad[v] = (grad[v] if accumulate) + scale * sum of grad_out[t] over the t with tokens[t] == v; none for skip_token."""
    if _table is None:
        _connect()
    _check(_calls.lmt_embed_grad(_table, grad_out, tokens, grad, workspace, scale, skip_token, accumulate, status, stream))


def fp8_shapes(rows: int, cols: int):
    """Shapes of the 8-bit form of a matrix and of its scales: ((rows, bytes of a row), (rows, bytes of a row's scales))."""
    return (rows, int(_lib().lmt_fp8_row_bytes(cols))), (rows, int(_lib().lmt_scale_row_bytes(cols)))


def quantize(x, q=None, scales=None, qt=None, scales_t=None, tile: bool = False, stream=None) -> None:
    """x [rows, cols] in 8 bits: q (float8_e4m3fn or float8_e5m2) and scales (uint8) of fp8_shapes(rows, cols), and / or the
    transpose, qt and scales_t of fp8_shapes(cols, rows); tile: one scale for a square of 128 x 128 instead of 128 elements."""
    if _table is None:
        _connect()
    _check(_calls.lmt_quantize(_table, x, q, scales, qt, scales_t, tile, stream))


def matmul_workspace(m: int, n: int, k: int) -> int:
    """Bytes of the uint8 tensor that matmul works in (0: none is needed)."""
    return int(_lib().lmt_matmul_workspace(m, n, k))


def matmul(a, a_scales, b, b_scales, c, workspace=None, accumulate: bool = False, stream=None, fp32_sums: bool = False) -> None:
    """c [m, n] = (c if accumulate) + a b^T for operands as quantize leaves them, of m and n rows.  fp32_sums: a 16-bit c from sums as exact as an fp32
    one's, at three to four fifths of the rate (lmt.h says what the others lose)."""
    if _table is None:
        _connect()
    _check(_calls.lmt_matmul(_table, a, a_scales, b, b_scales, c, workspace, accumulate, stream, fp32_sums))


def cross_entropy(logits, targets, loss=None, lse=None, grad=None, weights=None, ignore: int = -100, status=None, stream=None) -> None:
    """Per row: loss = w * (lse - logits[target]) and its gradient w * (softmax - onehot); see lmt.h for empty rows.
    loss, lse, weights: [rows] fp32 or None; grad: of the logits' type and shape, may be the logits, or None."""
    if _table is None:
        _connect()
    _check(_calls.lmt_cross_entropy(_table, logits, targets, loss, lse, grad, weights, ignore, status, stream))
