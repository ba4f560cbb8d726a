"""Rotary positions, attention and the loss of a product without a GPU: what the C entry points refuse, what the extension module hands on
or refuses, what is launched on a device that only notes it, and that the header is C."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import fake_device
import paper_2402_02447_amd as B
from paper_2402_02447_amd import lmt
from test_lmt_calls import F16, F32, I32, I64, BF, U8, Stream, Tensor

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                    # an address that nothing looks at
NULL, ARG, LIMIT, ALIGN, WORKSPACE = -1, -2, -3, -5, -6


def heads(h):
    return None if h is None else C.byref(lmt.Heads(*h))


def rotary(L, **c):
    a = dict(x=(P, 64, 16), dt=0, rows=5, heads=4, size=16, positions=P, ids=6, frequencies=P, pairs=8, magnitude=1.0, flags=0, out=(2 * P, 64, 16))
    a.update(c)
    a["x"], a["out"] = heads(a["x"]), heads(a["out"])
    return L.lmt_rotary(*a.values(), None)


BY = dict(dtype=2, flags=0, rows=5, heads=4, kv_heads=2, size=16, sequences=2, starts=P, lengths=None, prefixes=None, slopes=None, scale=1.0, cap=0.0, status=None)
WIDE, NARROW = (P, 64, 16), (P, 32, 16)


def attention(L, by=(), **c):
    a = dict(q=WIDE, k=NARROW, v=NARROW, out=WIDE, lse=P)
    a.update(c)
    return L.lmt_attention(None if by is None else C.byref(lmt.Attend(**dict(BY, **dict(by)))), *(heads(a[x]) for x in ("q", "k", "v", "out")), a["lse"], None)


def attention_grad(L, by=(), **c):
    a = dict(go=WIDE, q=WIDE, k=NARROW, v=NARROW, out=WIDE, lse=P, gq=WIDE, gk=NARROW, gv=NARROW, ws=P, ws_bytes=1 << 20)
    a.update(c)
    return L.lmt_attention_grad(None if by is None else C.byref(lmt.Attend(**dict(BY, **dict(by)))), *(heads(a[x]) for x in ("go", "q", "k", "v", "out")), a["lse"],
                                *(heads(a[x]) for x in ("gq", "gk", "gv")), a["ws"], a["ws_bytes"], None)


def loss(L, **c):
    a = dict(x=P, x_ld=8, table=P, table_ld=8, dt=2, rows=3, classes=7, width=8, t=P, ids=6, ignore=-100, w=None, loss=P, lse=P, gx=P, gx_ld=8, gt=P, gt_dt=2, gt_ld=8, flags=0, status=None,
             ws=P, ws_bytes=1 << 30)
    a.update(c)
    return L.lmt_linear_cross_entropy(*a.values(), None)


BAD = [
    (rotary, dict(x=None), NULL), (rotary, dict(x=(None, 64, 16)), NULL), (rotary, dict(out=None), NULL), (rotary, dict(positions=None), NULL), (rotary, dict(frequencies=None), NULL),
    (rotary, dict(dt=3), ARG), (rotary, dict(ids=0), ARG), (rotary, dict(flags=1), ARG), (rotary, dict(flags=32), ARG), (rotary, dict(magnitude=float("nan")), ARG), (rotary, dict(magnitude=1e39), ARG),
    (rotary, dict(pairs=9), ARG), (rotary, dict(out=(P, 64, 16), x=(P, 128, 16)), ARG), (rotary, dict(out=(2 * P, 63, 16)), ARG), (rotary, dict(out=(2 * P, 64, 15)), ARG), (rotary, dict(out=(2 * P, 16, 79)), ARG),
    (rotary, dict(size=129), LIMIT), (rotary, dict(heads=65536), LIMIT), (rotary, dict(rows=1 << 31), LIMIT), (rotary, dict(x=(P, 1 << 31, 16)), LIMIT), (rotary, dict(x=(P + 2, 64, 16)), ALIGN),
    (rotary, dict(out=(P + 1, 64, 16), dt=1), ALIGN), (rotary, dict(positions=P + 4), ALIGN), (rotary, dict(frequencies=P + 2), ALIGN)]
for call in (attention, attention_grad):
    BAD += [(call, dict(by=None), NULL), (call, dict(q=None), NULL), (call, dict(k=(None, 1, 1)), NULL), (call, dict(v=None), NULL), (call, dict(out=None), NULL), (call, dict(by=dict(starts=None)), NULL),
            (call, dict(by=dict(dtype=0)), ARG), (call, dict(by=dict(dtype=3)), ARG), (call, dict(by=dict(flags=1)), ARG), (call, dict(by=dict(prefixes=P)), ARG), (call, dict(by=dict(scale=float("inf"))), ARG),
            (call, dict(by=dict(scale=1e39)), ARG), (call, dict(by=dict(cap=-1.0)), ARG), (call, dict(by=dict(cap=float("nan"))), ARG), (call, dict(by=dict(cap=1e-40)), ARG), (call, dict(by=dict(cap=1e39)), ARG),
            (call, dict(by=dict(kv_heads=3)), ARG), (call, dict(by=dict(kv_heads=0)), ARG), (call, dict(by=dict(kv_heads=8)), ARG),
            (call, dict(by=dict(size=129)), LIMIT), (call, dict(by=dict(rows=1 << 31)), LIMIT), (call, dict(by=dict(sequences=1 << 31)), LIMIT), (call, dict(by=dict(heads=65536)), LIMIT),
            (call, dict(by=dict(rows=1 << 30, heads=32)), LIMIT), (call, dict(q=(P, 1 << 31, 16)), LIMIT), (call, dict(q=(P + 1, 64, 16)), ALIGN), (call, dict(lse=P + 2), ALIGN),
            (call, dict(by=dict(starts=P + 2)), ALIGN), (call, dict(by=dict(slopes=P + 1)), ALIGN), (call, dict(by=dict(lengths=P + 1)), ALIGN), (call, dict(by=dict(prefixes=P + 1, flags=32)), ALIGN),
            (call, dict(by=dict(status=P + 2)), ALIGN)]
BAD += [(attention, dict(out=(P, 63, 16)), ARG), (attention, dict(out=(P, 64, 0)), ARG), (attention, dict(out=(P, 0, 16)), ARG), (attention_grad, dict(gk=(P, 16, 16)), ARG), (attention_grad, dict(gq=(P, 60, 16)), ARG),
        (attention_grad, dict(gv=None), NULL), (attention_grad, dict(lse=None), NULL), (attention_grad, dict(go=None), NULL), (attention_grad, dict(ws=None), NULL), (attention_grad, dict(ws=P + 8), ALIGN),
        (attention_grad, dict(ws_bytes=64), WORKSPACE),
        (loss, dict(x=None), NULL), (loss, dict(table=None), NULL), (loss, dict(t=None), NULL), (loss, dict(ws=None), NULL), (loss, dict(dt=0), ARG), (loss, dict(dt=3), ARG), (loss, dict(ids=1), ARG),
        (loss, dict(gt_dt=1), ARG), (loss, dict(flags=2), ARG), (loss, dict(x_ld=7), ARG), (loss, dict(table_ld=7), ARG), (loss, dict(gx_ld=7), ARG), (loss, dict(gt_ld=7), ARG), (loss, dict(classes=0), ARG),
        (loss, dict(width=0), ARG), (loss, dict(rows=0), ARG), (loss, dict(rows=1 << 23), LIMIT), (loss, dict(classes=1 << 23), LIMIT), (loss, dict(width=1 << 23, x_ld=1 << 23, table_ld=1 << 23, gx_ld=1 << 23, gt_ld=1 << 23), LIMIT),
        (loss, dict(rows=1 << 22, classes=1 << 22), LIMIT), (loss, dict(x=P + 1), ALIGN), (loss, dict(gt=P + 2, gt_dt=0), ALIGN), (loss, dict(loss=P + 2), ALIGN), (loss, dict(t=P + 4), ALIGN), (loss, dict(ws=P + 8), ALIGN),
        (loss, dict(ws_bytes=100), WORKSPACE)]
for call in (attention, attention_grad):
    BAD += [(call, dict(by=dict(scale=3e38)), ARG), (call, dict(by=dict(scale=-3e38)), ARG), (call, dict(by=dict(cap=3e38)), ARG), (call, dict(by=dict(scale=1e20, cap=1e-20)), ARG),
            (call, dict(by=dict(heads=0)), ARG)]                                     # key heads that nobody asks would have gradients


@pytest.mark.parametrize("call,changed,code", BAD, ids=lambda x: getattr(x, "__name__", str(x)))
def test_the_c_entry_points_refuse(call, changed, code):
    L = lmt._lib()
    assert call(L, **changed) == code
    assert L.lmt_last_error()


def test_calls_with_nothing_to_do_succeed():
    L = lmt._lib()
    assert rotary(L, rows=0) == rotary(L, heads=0) == rotary(L, size=0, pairs=0) == 0
    assert attention(L, by=dict(rows=0), q=None) == attention(L, by=dict(heads=0, kv_heads=0)) == attention(L, by=dict(size=0)) == 0
    assert attention_grad(L, by=dict(rows=0), ws=None) == attention_grad(L, by=dict(size=0)) == 0
    assert loss(L, rows=0, gt=None, x=None) == loss(L, rows=0, flags=1) == loss(L, rows=0, classes=0) == 0
    assert lmt.attention_grad_workspace(0, 4, 2, 8) == lmt.attention_grad_workspace(5, 0, 0, 8) == lmt.attention_grad_workspace(5, 4, 2, 129) == 0
    assert lmt.linear_cross_entropy_workspace(0, 5, 5) == lmt.linear_cross_entropy_workspace(5, 0, 5) == lmt.linear_cross_entropy_workspace(1 << 23, 5, 5) == 0
    assert 0 < lmt.linear_cross_entropy_workspace(100, 500, 64, False) < lmt.linear_cross_entropy_workspace(100, 500, 64)


def test_frequencies():
    f = lmt.rotary_frequencies(4)
    assert f.dtype == F32 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001]))
    assert torch.allclose(lmt.rotary_frequencies(4, stretch=8.0), f / 8)
    g = lmt.rotary_frequencies(32, 10000.0, 4096, 4.0)
    plain = lmt.rotary_frequencies(32)
    turns = 4096 * plain / (2 * torch.pi)
    assert torch.equal(g[turns > 32.1], plain[turns > 32.1]) and torch.allclose(g[turns < 0.99], plain[turns < 0.99] / 4)
    between = (turns > 1.1) & (turns < 31)
    assert bool(between.any()) and bool((g < plain)[between].all()) and bool((g > plain / 4)[between].all())
    assert lmt.rotary_frequencies(0).numel() == 0


# ---- the extension module ---------------------------------------------------------------


@pytest.fixture(scope="module")
def module():
    L = lmt._lib()
    seen, keep, addresses = [], [], []

    def plain(x):
        if isinstance(x, C._Pointer):
            return tuple(getattr(x.contents, n) for n, _ in x.contents._fields_)
        return x
    for name in ("lmt_embed", "lmt_embed_grad", "lmt_quantize", "lmt_matmul", "lmt_cross_entropy", "lmt_linear_cross_entropy", "lmt_rotary", "lmt_attention", "lmt_attention_grad"):
        keep.append(C.CFUNCTYPE(C.c_int, *getattr(L, name).argtypes)(lambda *a: seen.append([plain(x) for x in a]) or 7))
        addresses.append(C.cast(keep[-1], C.c_void_p).value)
    from paper_2402_02447_amd import _calls as M
    types = {F32: 0, F16: 1, BF: 2, torch.float8_e4m3fn: 3, torch.float8_e5m2: 4, I32: 5, I64: 6, U8: 7}
    table = M.lmt_connect(*addresses, types, lambda: 0)
    few = M.lmt_connect(*addresses[:5], types, lambda: 0)

    def call(name, *args, of=table):
        seen.clear()
        rc = getattr(M, "lmt_" + name)(of, *args)
        return rc, seen[0]
    call.few = few
    yield call
    del keep


def T3(shape, dtype=BF, at=0x1000, stride=None, device=0):
    return Tensor(shape, dtype, at, stride or (shape[1] * shape[2], shape[2], 1), device)


ROTARY = [T3((5, 4, 16), F32, 0x10, (80, 20, 1)), Tensor((5,), I32, 0x20), Tensor((6,), F32, 0x30), T3((5, 4, 16), F32, 0x40, (16, 90, 1)), True, 1.5, True, None]
MASKS = [Tensor((3,), I32, 0x100), Tensor((2,), I32, 0x110), Tensor((2,), I32, 0x120), Tensor((4,), F32, 0x130), 0.5, 30.0, True, Tensor((1,), I32, 0x140), Stream()]
SEEN_MASKS = (2, 32, 5, 4, 2, 16, 2, 0x100, 0x110, 0x120, 0x130, 0.5, 30.0, 0x140)
ATTEND = [T3((5, 4, 16), BF, 0x10, (128, 16, 1)), T3((5, 2, 16), BF, 0x20, (128, 16, 1)), T3((5, 2, 16), BF, 0x30, (0, 16, 1)), T3((5, 4, 16), BF, 0x40), Tensor((4, 5), F32, 0x50), *MASKS]
GRAD = [T3((5, 4, 16), BF, 0x10), T3((5, 4, 16), BF, 0x20), T3((5, 2, 16), BF, 0x30), T3((5, 2, 16), BF, 0x40), T3((5, 4, 16), BF, 0x50), Tensor((4, 5), F32, 0x60), T3((5, 4, 16), BF, 0x70), T3((5, 2, 16), BF, 0x80),
        T3((5, 2, 16), BF, 0x90, (64, 16, 1)), Tensor((999,), U8, 0xA0), *MASKS]
LOSS = [Tensor((5, 8), BF, 0x10, (9, 1)), Tensor((7, 8), BF, 0x20), Tensor((5,), I64, 0x30), Tensor((999,), U8, 0x40), Tensor((5,), F32, 0x50), None, Tensor((5, 8), BF, 0x60), Tensor((7, 8), F32, 0x70, (10, 1)),
        Tensor((5,), F32, 0x80), -1, True, None, None]


def test_arguments_arrive_in_their_places(module):
    assert module("rotary", *ROTARY) == (7, [(0x10, 80, 20), 0, 5, 4, 16, 0x20, 5, 0x30, 6, 1.5, 8 + 16, (0x40, 16, 90), None])
    assert module("attention", *ATTEND) == (7, [SEEN_MASKS, (0x10, 128, 16), (0x20, 128, 16), (0x30, 0, 16), (0x40, 64, 16), 0x50, 0x7000_0000_1234])
    assert module("attention_grad", *GRAD) == (7, [SEEN_MASKS, (0x10, 64, 16), (0x20, 64, 16), (0x30, 32, 16), (0x40, 32, 16), (0x50, 64, 16), 0x60, (0x70, 64, 16), (0x80, 32, 16), (0x90, 64, 16), 0xA0, 999,
                                                   0x7000_0000_1234])
    assert module("linear_cross_entropy", *LOSS) == (7, [0x10, 9, 0x20, 8, 2, 5, 7, 8, 0x30, 6, -1, 0x80, 0x50, None, 0x60, 8, 0x70, 0, 10, 1, None, 0x40, 999, None])
    assert module("attention", *ATTEND[:4], None, Tensor((1,), I32, 0x100), None, None, None, 1.0, 0.0, False, None, 3)[1][0] == (2, 0, 5, 4, 2, 16, 0, 0x100, None, None, None, 1.0, 0.0, None)


def refused():
    for name, good, wrong in (
            ("rotary", ROTARY, {0: [None, Tensor((5, 64), F32), T3((5, 4, 16), F32, stride=(64, 32, 2)), T3((5, 4, 16), I32), T3((5, 4, 16), F32, device=-1), T3((4, 4, 16), F32)], 1: [Tensor((4,), I32), Tensor((5,), F32), None],
                                2: [None, Tensor((6,), F16), Tensor((6, 1), F32), Tensor((6,), F32, device=1)], 3: [None, T3((5, 4, 16), BF), T3((5, 4, 15), F32)]}),
            ("attention", ATTEND, {0: [None, T3((5, 4, 16), F32), T3((5, 4, 16), F16), T3((5, 4, 8)), T3((6, 4, 16))], 1: [T3((5, 2, 15)), T3((4, 2, 16)), T3((5, 2, 16), F16)], 2: [T3((5, 4, 16)), None],
                                   3: [T3((5, 2, 16)), T3((5, 4, 16), F32)], 4: [Tensor((5, 4), F32), Tensor((4, 5), BF), Tensor((4, 5), F32, stride=(6, 1)), Tensor((20,), F32)], 5: [None, Tensor((3,), I64), Tensor((0,), I32)],
                                   6: [Tensor((3,), I32), Tensor((2,), I64)], 7: [Tensor((3,), I32)], 8: [Tensor((2,), F32), Tensor((4,), BF)], 12: [Tensor((1,), I64)]}),
            ("attention_grad", GRAD, {0: [T3((5, 2, 16))], 4: [None], 5: [None, Tensor((4, 6), F32)], 6: [T3((5, 4, 16), F16)], 7: [T3((5, 4, 16))], 8: [None], 9: [Tensor((9,), I32)], 10: [None], 11: [Tensor((1,), I32)]}),
            ("linear_cross_entropy", LOSS, {0: [None, Tensor((5, 9), BF), Tensor((5, 8), F16)], 1: [Tensor((7, 9), BF)], 2: [Tensor((4,), I64)], 3: [Tensor((9,), F32)], 4: [Tensor((4,), F32)], 6: [Tensor((5, 8), F32)],
                                            7: [Tensor((7, 8), F16), Tensor((6, 8), BF)], 8: [Tensor((7,), F32)]})):
        for place, values in wrong.items():
            for n, x in enumerate(values):
                yield pytest.param(name, good[:place] + [x] + good[place + 1:], id=f"{name}-{place}-{n}")


@pytest.mark.parametrize("name,args", list(refused()))
def test_the_extension_module_refuses_what_does_not_fit(module, name, args):
    with pytest.raises(ValueError):
        module(name, *args)


def test_wrong_numbers_of_arguments_and_functions_that_are_not_there(module):
    for name, args in (("rotary", ROTARY), ("attention", ATTEND), ("attention_grad", GRAD), ("linear_cross_entropy", LOSS)):
        with pytest.raises(TypeError):
            module(name, 1)
        with pytest.raises(TypeError, match="without this function"):
            module(name, *args, of=module.few)
    from paper_2402_02447_amd import _calls as M
    with pytest.raises(TypeError):
        M.lmt_connect(1, 2, 3, 4, 5, 6, {}, lambda: 0)


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(3, 2, 4)
    with pytest.raises(ValueError, match="not on a GPU"):
        lmt.rotary(x, torch.zeros(3, dtype=torch.int64), torch.zeros(2), x)


# ---- launches ---------------------------------------------------------------------------

LIB = """
from ctypes import *
import os
L = CDLL(B.library_path())
for f in ("lmt_attention_grad_workspace", "lmt_linear_cross_entropy_workspace"):
    getattr(L, f).restype = c_uint64
P, U, D = (lambda x: c_void_p(x)), c_uint64, c_double
GB = 1 << 33
class H(Structure):
    _fields_ = [("at", c_void_p), ("row", c_uint64), ("head", c_uint64)]
class A(Structure):
    _fields_ = [("dtype", c_int32), ("flags", c_uint32)] + [(n, c_uint64) for n in ("rows", "heads", "kv_heads", "size", "sequences")] + [(n, c_void_p) for n in ("starts", "lengths", "prefixes", "slopes")] + [
        ("scale", c_double), ("cap", c_double), ("status", c_void_p)]
def h(heads, size):
    return byref(H(GB, heads * size, size))
def rotary(rows, heads, size, pairs, dt=2, out=2 * GB):
    return L.lmt_rotary(h(heads, size), dt, U(rows), U(heads), U(size), P(GB), 6, P(GB), U(pairs), D(1), 0, byref(H(out, heads * size, size)), None)
def attend(rows, heads, kv, size, grad=False, cap=0.0, dt=2):
    a = byref(A(dt, 0, rows, heads, kv, size, 3, GB, None, None, None, 1.0, cap, None))
    q, k = h(heads, size), h(kv, size)
    if not grad:
        return L.lmt_attention(a, q, k, k, q, P(GB), None)
    ws = L.lmt_attention_grad_workspace(U(rows), U(heads), U(kv), U(size))
    return L.lmt_attention_grad(a, q, q, k, k, q, P(GB), q, k, k, P(GB), U(ws), None)
def loss(rows, classes, width, gx=GB, gt=GB, gt_dt=2, dt=2, ld=None):
    ld = U(ld or width)
    ws = L.lmt_linear_cross_entropy_workspace(U(rows), U(classes), U(width), 1 if gx or gt else 0)
    return L.lmt_linear_cross_entropy(P(GB), ld, P(GB), ld, dt, U(rows), U(classes), U(width), P(GB), 6, c_int64(-100), None, P(GB), P(GB), P(gx), ld, P(gt), gt_dt, ld, 0, None, P(GB), U(ws), None)
"""


@pytest.fixture(scope="module")
def noted(tmp_path_factory):
    return fake_device.build(tmp_path_factory.mktemp("fake"))


def test_a_grid_never_has_more_threads_than_32_bits_count(noted):
    fake_device.run(noted, LIB + """
LIMIT = -3
most = {}
for call in (lambda: rotary(0x7fffff00, 1, 8, 4), lambda: rotary(1 << 24, 300, 128, 64), lambda: rotary(3, 65535, 128, 64), lambda: attend(0x3fffff80, 1, 1, 8), lambda: attend(0x3fffff80, 1, 1, 8, True),
             lambda: attend(1 << 20, 1000, 1000, 128), lambda: attend(1 << 20, 1000, 1, 128, True), lambda: attend(5, 65535, 5, 64, True), lambda: loss(0x7fffff, 60, 8), lambda: loss(60, 0x7fffff, 8),
             lambda: loss(64, 64, 0x7fffff), lambda: loss(180000, 180000, 64), lambda: loss(0x7fffff, 60, 8, None, None)):
    assert call() == 0
    seen = kernels()
    assert seen and all(0 < g and g * (512 if k.startswith("k_linear") else 256) < 1 << 32 for k, g in seen), seen
for call in (lambda: attend(0x7fffff00, 100, 1, 8), lambda: attend(0x7fffff00, 100, 1, 8, True), lambda: loss(0x7fffff, 0x7fffff, 8)):
    assert call() == LIMIT and not kernels()
""")


def test_what_a_call_enqueues(noted):
    """Few launches, no memory of its own, and none for empty work."""
    fake_device.run(noted, LIB + """
before = fake.fake_device_allocations()
def names(call):
    fake.fake_fail_host_allocations(1)
    code = call()
    fake.fake_fail_host_allocations(0)
    assert code == 0
    return [k for k, _ in kernels()]
assert names(lambda: rotary(37, 8, 64, 32)) == ["k_rotary"] and names(lambda: rotary(37, 8, 64, 0, out=GB)) == [] and names(lambda: rotary(0, 8, 64, 32)) == []
for size in (1, 64, 65, 128):
    for cap in (0.0, 5.0):
        for dt in (1, 2):
            assert names(lambda: attend(300, 4, 4, size, cap=cap, dt=dt)) == ["k_attend"]
            assert names(lambda: attend(300, 4, 4, size, True, cap, dt))[:2] == ["k_attend_grad_q", "k_attend_grad_kv"]
assert names(lambda: attend(0, 4, 4, 64)) == names(lambda: attend(0, 4, 4, 64, True)) == names(lambda: loss(0, 9, 9, gt=None)) == []
assert names(lambda: loss(100, 500, 64, None, None))[-2:] == ["k_linear", "k_linear_rows"]
both = names(lambda: loss(8192, 30522, 1024))
assert both.count("k_linear") == 1 + 3 * 2 and both[0] == "k_linear_begin", both        # two pieces of the classes, three products each
assert names(lambda: loss(100, 500, 64, gt=None)).count("k_linear") == 3 and names(lambda: loss(100, 500, 64, gx=None)).count("k_linear") == 3
assert fake.fake_device_allocations() == before
""")


def test_c99_program_builds_against_the_header_and_runs(tmp_path):
    (tmp_path / "check.c").write_text("""
#include <stdio.h>
#include <string.h>
#include "lmt.h"
int main(void) {
  float x[64] = {0};
  int32_t starts[2] = {0, 2};
  lmt_heads h = {x, 16, 8};
  lmt_attend a = {LMT_BF16, LMT_CAUSAL, 2, 2, 2, 8, 1, starts, NULL, NULL, NULL, 1.0, 0.0, NULL};
  a.kv_heads = 4;
  if (lmt_attention(&a, &h, &h, &h, &h, NULL, NULL) != LMT_ERR_ARG || !strstr(lmt_last_error(), "multiple")) return 1;
  if (lmt_attention_grad(&a, &h, &h, &h, &h, &h, x, &h, &h, &h, x, 0, NULL) != LMT_ERR_ARG) return 2;
  if (lmt_rotary(&h, LMT_F32, 2, 2, 8, x, LMT_I32, x, 5, 1.0, 0, &h, NULL) != LMT_ERR_ARG) return 3;
  if (lmt_linear_cross_entropy(x, 4, x, 4, LMT_F32, 1, 1, 4, x, LMT_I32, -1, NULL, x, x, NULL, 0, NULL, 0, 0, 0, NULL, NULL, 0, NULL) != LMT_ERR_ARG) return 4;
  if (lmt_attention_grad_workspace(2, 2, 2, 8) < 16 || lmt_linear_cross_entropy_workspace(2, 2, 2, 1) == 0) return 5;
  printf("sizes %d %d\\n", (int)sizeof(lmt_heads), (int)sizeof(lmt_attend));
  return 0;
}
""")
    lib, exe = B.library_path(), str(tmp_path / "check")
    libdir = os.path.dirname(lib)
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "check.c"), "-o", exe, "-L", libdir, "-l:libbca.so",
                    f"-Wl,-rpath,{libdir}", "-Wl,--allow-shlib-undefined"], check=True)
    env = dict(os.environ, LD_LIBRARY_PATH=os.path.join(os.path.dirname(torch.__file__), "lib") + ":" + os.environ.get("LD_LIBRARY_PATH", ""))
    r = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert r.returncode == 0 and r.stdout.split() == ["sizes", str(C.sizeof(lmt.Heads)), str(C.sizeof(lmt.Attend))], (r.returncode, r.stdout)
