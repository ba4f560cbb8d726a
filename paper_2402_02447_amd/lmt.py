"""The operators of a language model's training step in libbca.so (include/lmt.h): embedding lookup and its table's
gradient, 8-bit quantisation and products, cross entropy with its gradient, from logits or from what they are a product of; rotary
positions, and attention within the sequences of a batch with its gradient.

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
LMT_STATUS_BAD_TOKEN, LMT_STATUS_BAD_TARGET, LMT_STATUS_BAD_SEQUENCE = 1, 2, 4
LMT_ACCUMULATE, LMT_TILE_SCALES, LMT_FP32_SUMS, LMT_NEIGHBOURS, LMT_INVERSE, LMT_CAUSAL = 1, 2, 4, 8, 16, 32
LMT_MAX_ROWS, LMT_MAX_WIDTH, LMT_MAX_HEAD, LMT_MAX_HEADS = 0x7FFFFF00, 0x7FFFFF, 128, 65535
_ERR = {-1: "LMT_ERR_NULL", -2: "LMT_ERR_ARG", -3: "LMT_ERR_LIMIT", -4: "LMT_ERR_HIP", -5: "LMT_ERR_ALIGN", -6: "LMT_ERR_WORKSPACE"}
_BYTES = 7                          # uint8: scales and workspaces

EXPORTS = ["lmt_embed", "lmt_embed_grad", "lmt_embed_grad_workspace", "lmt_fp8_row_bytes", "lmt_scale_row_bytes",
           "lmt_quantize", "lmt_matmul_workspace", "lmt_matmul", "lmt_cross_entropy", "lmt_last_error",
           "lmt_linear_cross_entropy_workspace", "lmt_linear_cross_entropy_workspace_of", "lmt_linear_cross_entropy", "lmt_rotary", "lmt_attention", "lmt_attention_grad_workspace", "lmt_attention_grad"]


class Heads(C.Structure):
    """lmt_heads: rows of heads, strides in elements."""
    _fields_ = [("at", C.c_void_p), ("row", C.c_uint64), ("head", C.c_uint64)]


class Attend(C.Structure):
    """lmt_attend: what attention goes by."""
    _fields_ = [("dtype", C.c_int32), ("flags", C.c_uint32), ("rows", C.c_uint64), ("heads", C.c_uint64), ("kv_heads", C.c_uint64), ("size", C.c_uint64),
                ("sequences", C.c_uint64), ("starts", C.c_void_p), ("lengths", C.c_void_p), ("prefixes", C.c_void_p), ("slopes", C.c_void_p),
                ("scale", C.c_double), ("cap", C.c_double), ("status", C.c_void_p)]


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
        heads, attend = C.POINTER(Heads), C.POINTER(Attend)
        L.lmt_linear_cross_entropy.argtypes = [vp, u64, vp, u64, i32, u64, u64, u64, vp, i32, i64, vp, vp, vp, vp, u64, vp, i32, u64, u32, vp, vp, u64, vp]
        L.lmt_rotary.argtypes = [heads, i32, u64, u64, u64, vp, i32, vp, u64, dbl, u32, heads, vp]
        L.lmt_attention.argtypes = [attend, heads, heads, heads, heads, vp, vp]
        L.lmt_attention_grad.argtypes = [attend] + 5 * [heads] + [vp] + 3 * [heads] + [vp, u64, vp]
        L.lmt_linear_cross_entropy_workspace.argtypes, L.lmt_linear_cross_entropy_workspace.restype = [u64, u64, u64, i32], u64
        L.lmt_linear_cross_entropy_workspace_of.argtypes, L.lmt_linear_cross_entropy_workspace_of.restype = [i32, u64, u64, u64, i32], u64
        L.lmt_attention_grad_workspace.argtypes, L.lmt_attention_grad_workspace.restype = [u64, u64, u64, u64], u64
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
    addresses = [C.cast(getattr(L, f), C.c_void_p).value for f in ("lmt_embed", "lmt_embed_grad", "lmt_quantize", "lmt_matmul", "lmt_cross_entropy",
                                                                        "lmt_linear_cross_entropy", "lmt_rotary", "lmt_attention", "lmt_attention_grad")]
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


def linear_cross_entropy_workspace(rows: int, classes: int, width: int, gradients: bool = True, dtype=None) -> int:
    """Bytes of the uint8 tensor that linear_cross_entropy works in, with or without gradients: enough for any call of these sizes, or with dtype
    (torch.float16 or torch.bfloat16) what a call of this type needs whose x and table start on 16 bytes, with row strides of whole 16 bytes, as new tensors do."""
    if dtype is None:
        return int(_lib().lmt_linear_cross_entropy_workspace(rows, classes, width, gradients))
    import torch
    if dtype not in (torch.float16, torch.bfloat16):
        raise ValueError("dtype: fp16 or bf16 is wanted")
    return int(_lib().lmt_linear_cross_entropy_workspace_of(LMT_F16 if dtype == torch.float16 else LMT_BF16, rows, classes, width, gradients))


def linear_cross_entropy(x, table, targets, workspace, loss=None, lse=None, grad_x=None, grad_table=None, weights=None, ignore: int = -100,
                         accumulate: bool = False, status=None, stream=None) -> None:
    """cross_entropy of the logits x table^T, which are not kept, with the gradients of x and of the table (added to
    grad_table with accumulate).  x: [rows, width], table: [classes, width], fp16 or bf16; grad_x: as x; grad_table: as the table, or fp32;
    each result may be None."""
    if _table is None:
        _connect()
    _check(_calls.lmt_linear_cross_entropy(_table, x, table, targets, workspace, loss, lse, grad_x, grad_table, weights, ignore, accumulate, status, stream))


def rotary_frequencies(pairs: int, base: float = 10000.0, trained: int = 0, stretch: float = 1.0, kept: float = 32.0, slowed: float = 1.0):
    """Frequencies (fp32, on the host) of `pairs` pairs of a head, base^(-f / pairs), for contexts `stretch` times as long as the `trained` positions.
    A pair that makes `kept` turns or more within `trained` positions keeps its frequency, one that makes `slowed` or fewer is slowed by
    `stretch`, those between by as much as lies between (the published interpolation of rotary frequencies by parts); with trained = 0 all are slowed."""
    import math

    import torch
    f = float(base) ** (-torch.arange(pairs, dtype=torch.float64) / max(1, pairs))
    keep = ((trained * f / (2 * math.pi) - slowed) / (kept - slowed)).clamp(0, 1) if trained else torch.zeros_like(f)
    return (f * (keep + (1 - keep) / stretch)).float()


def rotary(x, positions, frequencies, out, neighbours: bool = False, magnitude: float = 1.0, inverse: bool = False, stream=None) -> None:
    """The first pairs of every head turned by position * frequency and multiplied by `magnitude`, the rest copied; inverse: turned back, which with
    the same magnitude is the gradient.  x, out: [rows, heads, size] with any strides between rows and heads, out may be x; positions: [rows] int32
    or int64; frequencies: [pairs] fp32, radians; neighbours: pairs are neighbours instead of `pairs` elements apart."""
    if _table is None:
        _connect()
    _check(_calls.lmt_rotary(_table, x, positions, frequencies, out, neighbours, magnitude, inverse, stream))


def attention(q, k, v, out, lse, starts, lengths=None, prefixes=None, slopes=None, scale: float = 1.0, cap: float = 0.0, causal: bool = False,
              status=None, stream=None) -> None:
    """out = softmax(scores) v for every row within its sequence.  q, out: [rows, heads, size], k, v: [rows, kv_heads, size], fp16 or bf16, with any
    strides between rows and heads; lse: [heads, rows] fp32 or None; starts: int32, where each sequence begins and the last one ends; lengths:
    int32, where sequences end before the next one begins, or None; causal: none sees later positions, but for the first prefixes[s] of its sequence;
    scores are scale * q.k, then cap * tanh(scores / cap) if there is a cap, then - slopes[head] * distance.  Rows of no sequence get
    zeros and -inf.  status: int32 or None (LMT_STATUS_BAD_SEQUENCE)."""
    if _table is None:
        _connect()
    _check(_calls.lmt_attention(_table, q, k, v, out, lse, starts, lengths, prefixes, slopes, scale, cap, causal, status, stream))


def attention_grad_workspace(rows: int, heads: int, kv_heads: int, size: int) -> int:
    """Bytes of the uint8 tensor that attention_grad works in."""
    return int(_lib().lmt_attention_grad_workspace(rows, heads, kv_heads, size))


def attention_grad(grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, workspace, starts, lengths=None, prefixes=None, slopes=None, scale: float = 1.0,
                   cap: float = 0.0, causal: bool = False, status=None, stream=None) -> None:
    """Gradients of attention's q, k and v from that of out; out and lse are what attention left, the rest what it was given."""
    if _table is None:
        _connect()
    _check(_calls.lmt_attention_grad(_table, grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, workspace, starts, lengths, prefixes, slopes, scale, cap, causal, status, stream))
