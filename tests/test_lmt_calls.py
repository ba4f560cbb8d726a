"""lmt.h without a GPU: what the C entry points refuse, and what the extension module hands on or refuses, with functions
that note what they are given."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2402_02447_amd import lmt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                    # an address that nothing looks at


def test_exports_errors_and_constants_agree_with_the_header():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lmt.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(lmt_[a-z0-9_]+)\s*\(", header)) == set(lmt.EXPORTS)
    defines = {k: int(v, 0) for k, v in re.findall(r"#define (LMT_[A-Z0-9_]+) \(?(-?(?:0x)?[0-9a-f]+)u?\)?", header)}
    for name, value in defines.items():
        if "_ERR_" in name:
            assert lmt._ERR[value] == name
        elif name != "LMT_H_":
            assert getattr(lmt, name) == value, name
    assert len(lmt._ERR) == sum("_ERR_" in k for k in defines)


def embed(L, **c):
    a = dict(table=P, dt=0, vocab=10, width=8, table_ld=8, tokens=P, ids=5, n=3, scale=1.0, out=P, odt=0, out_ld=8, status=None)
    a.update(c)
    return L.lmt_embed(*a.values(), None)


def grad(L, **c):
    a = dict(go=P, dt=0, go_ld=8, tokens=P, ids=6, n=3, scale=1.0, skip=-1, g=P, gdt=0, vocab=10, width=8, g_ld=8, flags=0, status=None, ws=P, ws_bytes=1 << 30)
    a.update(c)
    return L.lmt_embed_grad(*a.values(), None)


def quantize(L, **c):
    a = dict(x=P, dt=0, rows=5, cols=9, ld=9, fp8=3, flags=0, q=P, s=P, qt=P, st=P)
    a.update(c)
    return L.lmt_quantize(*a.values(), None)


def matmul(L, **c):
    a = dict(a=P, af=3, a_s=P, b=P, bf=4, b_s=P, m=3, n=4, k=5, c=P, cdt=0, ldc=4, flags=0, ws=P, ws_bytes=1 << 40)
    a.update(c)
    return L.lmt_matmul(*a.values(), None)


def loss(L, **c):
    a = dict(x=P, dt=0, rows=3, classes=7, ld=7, t=P, ids=5, ignore=-100, w=None, loss=P, lse=P, grad=P + 4096, g_ld=7, status=None)
    a.update(c)
    return L.lmt_cross_entropy(*a.values(), None)


NULL, ARG, LIMIT, ALIGN, WORKSPACE = -1, -2, -3, -5, -6
REFUSED = [
    (embed, dict(table=None), NULL), (embed, dict(tokens=None), NULL), (embed, dict(out=None), NULL), (embed, dict(dt=3), ARG), (embed, dict(odt=7), ARG),
    (embed, dict(ids=0), ARG), (embed, dict(scale=float("nan")), ARG), (embed, dict(scale=1e39), ARG), (embed, dict(table_ld=7), ARG), (embed, dict(out_ld=7), ARG),
    (embed, dict(vocab=1 << 31), LIMIT), (embed, dict(n=1 << 31), LIMIT), (embed, dict(width=1 << 23, table_ld=1 << 23, out_ld=1 << 23), LIMIT),
    (embed, dict(table=P + 2), ALIGN), (embed, dict(out=P + 1, odt=1), ALIGN), (embed, dict(tokens=P + 4, ids=6), ALIGN), (embed, dict(status=P + 1), ALIGN),
    (grad, dict(go=None), NULL), (grad, dict(tokens=None), NULL), (grad, dict(g=None), NULL), (grad, dict(ws=None), NULL), (grad, dict(dt=5), ARG), (grad, dict(gdt=-1), ARG),
    (grad, dict(ids=3), ARG), (grad, dict(flags=2), ARG), (grad, dict(scale=float("inf")), ARG), (grad, dict(go_ld=1), ARG), (grad, dict(g_ld=1), ARG),
    (grad, dict(vocab=1 << 31), LIMIT), (grad, dict(n=1 << 31), LIMIT), (grad, dict(ws=P + 8), ALIGN), (grad, dict(g=P + 2), ALIGN), (grad, dict(tokens=P + 4), ALIGN),
    (grad, dict(ws_bytes=0), WORKSPACE), (grad, dict(ws_bytes=100), WORKSPACE),
    (quantize, dict(x=None), NULL), (quantize, dict(s=None), NULL), (quantize, dict(q=None), NULL), (quantize, dict(st=None), NULL),
    (quantize, dict(q=None, s=None, qt=None, st=None), NULL), (quantize, dict(dt=4), ARG), (quantize, dict(fp8=2), ARG), (quantize, dict(flags=1), ARG), (quantize, dict(ld=8), ARG),
    (quantize, dict(rows=1 << 31), LIMIT), (quantize, dict(cols=1 << 23, ld=1 << 23), LIMIT), (quantize, dict(rows=1 << 23), LIMIT), (quantize, dict(x=P + 2), ALIGN),
    (quantize, dict(q=P + 8), ALIGN), (quantize, dict(qt=P + 4), ALIGN),
    (matmul, dict(a=None), NULL), (matmul, dict(a_s=None), NULL), (matmul, dict(b=None), NULL), (matmul, dict(b_s=None), NULL), (matmul, dict(c=None), NULL),
    (matmul, dict(af=2), ARG), (matmul, dict(bf=5), ARG), (matmul, dict(cdt=3), ARG), (matmul, dict(flags=2), ARG), (matmul, dict(ldc=3), ARG), (matmul, dict(k=1 << 23), LIMIT),
    (matmul, dict(m=1 << 31), LIMIT), (matmul, dict(a=P + 8), ALIGN), (matmul, dict(b=P + 1), ALIGN), (matmul, dict(a_s=P + 2), ALIGN), (matmul, dict(c=P + 2), ALIGN),
    (matmul, dict(m=64, n=64, k=1 << 20, ldc=64, ws=None), NULL), (matmul, dict(m=64, n=64, k=1 << 20, ldc=64, ws_bytes=16), WORKSPACE),
    (loss, dict(x=None), NULL), (loss, dict(t=None), NULL), (loss, dict(dt=3), ARG), (loss, dict(ids=1), ARG), (loss, dict(ld=6), ARG), (loss, dict(g_ld=6), ARG),
    (loss, dict(classes=0), ARG), (loss, dict(grad=P, g_ld=8), ARG), (loss, dict(rows=1 << 31), LIMIT), (loss, dict(classes=1 << 31, ld=1 << 31, g_ld=1 << 31), LIMIT),
    (loss, dict(x=P + 2), ALIGN), (loss, dict(loss=P + 2), ALIGN), (loss, dict(w=P + 1), ALIGN), (loss, dict(t=P + 4, ids=6), ALIGN),
]


@pytest.mark.parametrize("call,changed,code", REFUSED, ids=lambda x: getattr(x, "__name__", str(x)))
def test_the_c_entry_points_refuse(call, changed, code):
    L = lmt._lib()
    assert call(L, **changed) == code
    assert L.lmt_last_error()


def test_calls_with_nothing_to_do_succeed():
    L = lmt._lib()
    assert embed(L, n=0, tokens=None, out=None) == 0 and embed(L, width=0) == 0
    assert grad(L, vocab=0) == 0 and grad(L, width=0) == 0 and grad(L, n=0, flags=1, go=None, tokens=None, ws=None) == 0
    assert quantize(L, rows=0) == 0 and quantize(L, cols=0) == 0
    assert matmul(L, m=0) == 0 and matmul(L, n=0) == 0 and matmul(L, k=0, flags=1) == 0
    assert loss(L, rows=0, x=None, t=None) == 0
    assert lmt.embed_grad_workspace(0, 5, 5) == lmt.embed_grad_workspace(5, 0, 5) == lmt.embed_grad_workspace(5, 5, 0) == 0
    assert lmt.matmul_workspace(0, 5, 5) == lmt.matmul_workspace(5, 0, 5) == 0
    assert lmt.fp8_shapes(3, 0) == ((3, 0), (3, 0)) and lmt.fp8_shapes(3, 1) == ((3, 128), (3, 4)) and lmt.fp8_shapes(2, 513) == ((2, 640), (2, 8))


def test_the_workspace_of_a_product_is_that_of_its_operands_blocks():
    """Operands do not say how much of their last block is padding."""
    for m, n in ((1, 64), (37, 1024), (65, 300), (300, 1000), (2432, 30522), (4096, 1024)):
        for k in (1, 100, 128, 129, 1000, 1023, 1025, 4000, 4095, 5000, 16380, 32700):
            assert lmt.matmul_workspace(m, n, k) == lmt.matmul_workspace(m, n, -(-k // 128) * 128), (m, n, k)


# ---- the extension module ---------------------------------------------------------------


class Tensor:
    """What the module looks at of a tensor."""

    def __init__(self, shape, dtype, at=0x1000, stride=None, device=0):
        self.shape, self.dtype, self.at, self.device = tuple(shape), dtype, at, device
        self._stride = tuple(stride) if stride else ((shape[1], 1) if len(shape) == 2 else (1,) * len(shape))

    def data_ptr(self):
        return self.at

    def stride(self):
        return self._stride

    def get_device(self):
        return self.device


F32, F16, BF, E4, E5, I32, I64, U8 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2, torch.int32, torch.int64, torch.uint8


@pytest.fixture(scope="module")
def module():
    L = lmt._lib()
    seen, keep, addresses = [], [], []
    for name in ("lmt_embed", "lmt_embed_grad", "lmt_quantize", "lmt_matmul", "lmt_cross_entropy"):
        keep.append(C.CFUNCTYPE(C.c_int, *getattr(L, name).argtypes)(lambda *a: seen.append(list(a)) or 7))
        addresses.append(C.cast(keep[-1], C.c_void_p).value)
    from paper_2402_02447_amd import _calls as M
    types = {F32: 0, F16: 1, BF: 2, E4: 3, E5: 4, I32: 5, I64: 6, U8: 7}
    table = M.lmt_connect(*addresses, types, lambda: 0)

    def call(name, *args):
        seen.clear()
        rc = getattr(M, "lmt_" + name)(table, *args)
        return rc, seen[0]
    yield call
    del keep


class Stream:
    cuda_stream = 0x7000_0000_1234


def test_arguments_arrive_in_their_places(module):
    assert module("embed", Tensor((9, 6), F16, 0x10, (8, 1)), Tensor((4,), I32, 0x20), Tensor((4, 6), F32, 0x30, (7, 1)), 2.5, Tensor((1,), I32, 0x40), Stream()) == (
        7, [0x10, 1, 9, 6, 8, 0x20, 5, 4, 2.5, 0x30, 0, 7, 0x40, 0x7000_0000_1234])
    assert module("embed_grad", Tensor((4, 6), BF, 0x10, (9, 1)), Tensor((4,), I64, 0x20), Tensor((11, 6), F32, 0x30), Tensor((99,), U8, 0x50), 0.5, -7, True, None, None) == (
        7, [0x10, 2, 9, 0x20, 6, 4, 0.5, -7, 0x30, 0, 11, 6, 6, 1, None, 0x50, 99, None])
    x, q, s, t, ts = Tensor((130, 5), F32, 0x10), Tensor((130, 128), E5, 0x20), Tensor((130, 4), U8, 0x30), Tensor((5, 256), E5, 0x40), Tensor((5, 4), U8, 0x50)
    assert module("quantize", x, q, s, t, ts, True, 5) == (7, [0x10, 0, 130, 5, 5, 4, 2, 0x20, 0x30, 0x40, 0x50, 5])
    assert module("quantize", x, None, None, t, ts, False, None) == (7, [0x10, 0, 130, 5, 5, 4, 0, None, None, 0x40, 0x50, None])
    a, a_s, b, b_s = Tensor((3, 640), E4, 0x10), Tensor((3, 8), U8, 0x20), Tensor((9, 640), E5, 0x30), Tensor((9, 8), U8, 0x40)
    assert module("matmul", a, a_s, b, b_s, Tensor((3, 9), BF, 0x60, (12, 1)), Tensor((64,), U8, 0x70), True, None) == (
        7, [0x10, 3, 0x20, 0x30, 4, 0x40, 3, 9, 640, 0x60, 2, 12, 1, 0x70, 64, None])
    assert module("cross_entropy", Tensor((2, 50), BF, 0x10, (64, 1)), Tensor((2,), I64, 0x20), Tensor((2,), F32, 0x30), None, Tensor((2, 50), BF, 0x40), Tensor((2,), F32, 0x50), -1, None, None) == (
        7, [0x10, 2, 2, 50, 64, 0x20, 6, -1, 0x50, 0x30, None, 0x40, 50, None, None])
    # one row: whatever its stride is
    assert module("embed", Tensor((1, 6), F32, 0x10, (1, 1)), Tensor((1,), I32, 0x20, (5,)), Tensor((1, 6), F32, 0x30, (0, 1)), 1.0, None, None)[1][2:5] == [1, 6, 6]


def refused():
    e = [Tensor((9, 6), F32), Tensor((4,), I32), Tensor((4, 6), F32), 1.0, None, None]
    g = [Tensor((4, 6), F32), Tensor((4,), I32), Tensor((9, 6), F32), Tensor((99,), U8), 1.0, -1, False, None, None]
    q = [Tensor((130, 5), F32), Tensor((130, 128), E4), Tensor((130, 4), U8), Tensor((5, 256), E4), Tensor((5, 4), U8), False, None]
    m = [Tensor((3, 640), E4), Tensor((3, 8), U8), Tensor((9, 640), E4), Tensor((9, 8), U8), Tensor((3, 9), F32), None, False, None]
    c = [Tensor((2, 50), F32), Tensor((2,), I64), Tensor((2,), F32), None, Tensor((2, 50), F32), None, -1, None, None]
    for name, good, place, wrong in (
            [("embed", e, 0, x) for x in (None, Tensor((54,), F32), Tensor((9, 6), F32, stride=(12, 2)), Tensor((9, 6), F32, stride=(5, 1)), Tensor((9, 6), F32, stride=(0, 1)), Tensor((9, 6), E4), Tensor((9, 6), torch.float64), Tensor((9, 6), F32, device=-1), Tensor((9, 7), F32))]
            + [("embed", e, 1, x) for x in (None, Tensor((4, 1), I32), Tensor((4,), F32), Tensor((5,), I32), Tensor((4,), I32, stride=(2,)), Tensor((4,), I32, device=1))]
            + [("embed", e, 2, Tensor((4, 5), F32)), ("embed", e, 4, Tensor((1,), I64)), ("embed", e, 4, Tensor((0,), I32))]
            + [("embed_grad", g, 0, Tensor((3, 6), F32)), ("embed_grad", g, 2, Tensor((9, 5), F32)), ("embed_grad", g, 3, Tensor((99,), I32)), ("embed_grad", g, 3, Tensor((9, 11), U8))]
            + [("quantize", q, 1, x) for x in (Tensor((130, 128), F16), Tensor((130, 256), E4), Tensor((129, 128), E4), Tensor((130, 128), E4, stride=(129, 1)), Tensor((130, 128), E5), None)]
            + [("quantize", q, 2, x) for x in (Tensor((130, 5), U8), Tensor((130, 4), I32), Tensor((130, 4), U8, stride=(8, 1)), None)]
            + [("quantize", q, 3, Tensor((5, 128), E4)), ("quantize", q, 4, None)]
            + [("matmul", m, 0, x) for x in (None, Tensor((3, 641), E4), Tensor((3, 512), E4), Tensor((3, 640), BF), Tensor((4, 640), E4))]
            + [("matmul", m, 1, None), ("matmul", m, 1, Tensor((3, 5), U8)), ("matmul", m, 4, Tensor((9, 3), F32)), ("matmul", m, 4, Tensor((3, 9), E4)), ("matmul", m, 5, Tensor((9,), F32))]
            + [("cross_entropy", c, 1, Tensor((3,), I64)), ("cross_entropy", c, 2, Tensor((3,), F32)), ("cross_entropy", c, 2, Tensor((2,), BF)), ("cross_entropy", c, 4, Tensor((2, 50), BF)),
               ("cross_entropy", c, 4, Tensor((2, 49), F32)), ("cross_entropy", c, 5, Tensor((1,), F32))]):
        yield pytest.param(name, good[:place] + [wrong] + good[place + 1:], id=f"{name}-{place}-{getattr(wrong, 'shape', wrong)}-{getattr(wrong, 'dtype', '')}")


@pytest.mark.parametrize("name,args", list(refused()))
def test_the_extension_module_refuses_what_does_not_fit(module, name, args):
    with pytest.raises(ValueError):
        module(name, *args)


def test_wrong_numbers_of_arguments_and_kinds(module):
    for name in ("embed", "embed_grad", "quantize", "matmul", "cross_entropy"):
        with pytest.raises(TypeError):
            module(name, 1)
    with pytest.raises(AttributeError):
        module("embed", object(), Tensor((4,), I32), Tensor((4, 6), F32), 1.0, None, None)
    with pytest.raises(TypeError):
        module("embed", Tensor((9, 6), F32), Tensor((4,), I32), Tensor((4, 6), F32), "much", None, None)


def test_tensors_on_the_host_are_refused():
    with pytest.raises(ValueError, match="not on a GPU"):
        lmt.embed(torch.zeros(3, 4), torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4))
