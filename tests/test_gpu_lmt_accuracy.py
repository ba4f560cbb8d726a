"""How exact products are (GPU): sums seen through 16-bit results, in norms instead of worst cases, and 16-bit results from fp32 sums."""
import numpy as np
import pytest
import torch

import lmt_reference as R
from lmt_gpu import DT, Mat, typed
from paper_2402_02447_amd import lmt
from test_gpu_lmt_fp8 import F8, SIZES, operand, put

pytestmark = pytest.mark.gpu


def product(a, b, c, accumulate=False, fp32_sums=False):
    need = lmt.matmul_workspace(a[0].shape[0], b[0].shape[0], a[0].shape[1])
    ws = torch.full((need + 64,), 0x77, dtype=torch.uint8, device="cuda")
    lmt.matmul(*a, *b, c, ws[:need], accumulate, fp32_sums=fp32_sums)
    assert bool((ws[need:] == 0x77).all())


# ---- 16-bit results from fp32 sums ---------------------------------------------------------


def check_same_as_fp32(m, n, k, af, bf, kind, accumulate, seed):
    """The sums are those of an fp32 result, which has a test of its own; what differs is the one rounding at the end."""
    rng = np.random.default_rng(seed)
    a, b = operand(rng, m, k, af), operand(rng, n, k, bf)
    old = typed(rng.normal(0, 10, (m, n)), kind)
    if kind == "f16":                                             # in range, most of them
        for (q, s), form in ((a, af), (b, bf)):
            s[:, :q.shape[1] // 128] = 127 - (4 if form == R.E4M3 else 12)
    a, b = put(*a, af), put(*b, bf)
    c, wide = Mat(m, n, kind, 3, 1, old), torch.tensor(old, dtype=torch.float32, device="cuda")
    product(a, b, c.view, accumulate, True)
    product(a, b, wide, accumulate)
    assert torch.equal(c.view, wide.to(DT[kind])) and c.untouched_outside()


@pytest.mark.parametrize("af", [R.E4M3, R.E5M2])
@pytest.mark.parametrize("bf", [R.E4M3, R.E5M2])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_fp32_sums_of_every_type(af, bf, kind, accumulate):
    for m, n, k in ((40, 90, 300), (70, 90, 300), (64, 100, 8192)):
        check_same_as_fp32(m, n, k, af, bf, kind, accumulate, 1)
    check_same_as_fp32(4096, 4096, 256, af, bf, kind, accumulate, 2)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_fp32_sums_of_every_size(m, n, k):
    check_same_as_fp32(m, n, k, R.E4M3, R.E5M2, "bf16", True, m)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_fp32_sums_say_nothing_to_an_fp32_result_and_to_none(kind):
    a, b = (torch.empty(r, 0, dtype=torch.float8_e4m3fn, device="cuda") for r in (3, 5))
    s, t = (torch.empty(r, 0, dtype=torch.uint8, device="cuda") for r in (3, 5))
    c = torch.ones(3, 5, dtype=DT[kind], device="cuda")
    lmt.matmul(a, s, b, t, c, fp32_sums=True)
    assert (c == 0).all()


# ---- norms ---------------------------------------------------------------------------------

SHAPES = [(40, 512, 1024), (300, 512, 1024), (4096, 4096, 1024), (512, 512, 16384)]   # few rows; tiles of both sizes; k in parts


def quantised(x, form):
    q, s = (torch.empty(n, dtype=t, device="cuda") for n, t in zip(lmt.fp8_shapes(*x.shape), (F8[form], torch.uint8)))
    lmt.quantize(x, q, s)
    return (q, s), torch.ldexp(q.double().view(x.shape[0], -1, 128), (s[:, :q.shape[1] // 128].int() - 127).unsqueeze(2)).view(x.shape[0], -1)


def sums(m, n, k, form, numbers, kind, fp32_sums=False):
    """Errors of a product's sums, and the exact ones.  A 16-bit result shows its sum when it is added to the negative of the sum's rounding: what
    is left is small, so that its own rounding (2^-11 of 2^-11) does not hide the sum's error."""
    g = torch.Generator(device="cuda")
    g.manual_seed(k)
    x, y = (torch.randn(r, k, generator=g, device="cuda") for r in (m, n))
    if numbers == "positive":
        x, y = x.abs(), y.abs()
    if numbers == "spread":
        x, y = (v * torch.exp(2 * torch.randn(v.shape, generator=g, device="cuda")) for v in (x, y))
    x *= {"positive": 1000 / 0.64 / k, "normal": 1000 / k ** 0.5, "spread": 20 / k ** 0.5}[numbers]      # results of about 1 000, and what fp16 still holds
    a, A = quantised(x, form)
    b, B = quantised(y, R.E4M3)
    exact = torch.mm(A, B.t().contiguous())
    if kind == "f32":
        c = torch.empty(m, n, device="cuda")
        product(a, b, c)
        return c.double() - exact, exact
    near = exact.clamp(-60000, 60000).half()
    c = -near
    product(a, b, c, True, fp32_sums)
    error = c.double() - (exact - near.double())
    return torch.where(exact.abs() < 60000, error, 0.0), exact


# of the result's 2-norm.  8-bit instructions: what lmt.h states, and half of it for the draw
NARROW = {"normal": 1.5 * 1.5e-5, "spread": 1.5 * 4e-5, "positive": 1.5 * 3e-6 + 2.0 ** -20}


def wide_bound(k, numbers):
    """fp32 sums of k terms: at most one rounding for eight of them (the least that an instruction takes), each uniform within u of the partial sum, so
    u / sqrt(3) times the root of the sum of the partial sums' squares, which grow as the root of the terms so far, or as the terms if all are positive.
    Numbers that spread have partial sums as large as the whole from the first large term on.  Twice that; and 2^-22 for what an fp16 result shows."""
    n = max(k / 8, 1)
    return 2 * R.U32 / 3 ** 0.5 * {"normal": (n / 2) ** 0.5, "positive": (n / 3) ** 0.5, "spread": n ** 0.5}[numbers] + 2.0 ** -22


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("numbers", ["normal", "spread", "positive"])
@pytest.mark.parametrize("form", [R.E4M3, R.E5M2])
def test_norm_of_the_errors_of_sums(m, n, k, numbers, form):
    for kind, fp32_sums in (("f16", False), ("f16", True), ("f32", False)):
        error, exact = sums(m, n, k, form, numbers, kind, fp32_sums)
        got = float(error.norm() / exact.norm())
        assert got <= (wide_bound(k, numbers) if fp32_sums or kind == "f32" else NARROW[numbers]), (kind, fp32_sums, got)


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_sums_of_one_sign_do_not_drift(m, n, k):
    """An accumulator that cut digits off would lose in proportion to k.  The 8-bit instructions cut off 3e-6 of what they add, once; roundings to
    nearest have no mean beside their random one, over m n results."""
    for kind, fp32_sums, bound in (("f16", False, 1.5 * 3e-6), ("f16", True, 3e-7), ("f32", False, 3e-7)):
        error, exact = sums(m, n, k, R.E4M3, "positive", kind, fp32_sums)
        assert abs(float(error.mean() / exact.mean())) <= bound, (kind, fp32_sums)


@pytest.mark.parametrize("m", [8, 100])
@pytest.mark.parametrize("kind,fp32_sums", [("f32", False), ("bf16", True), ("bf16", False)])
def test_scales_at_their_ends(m, kind, fp32_sums):
    """Codes times the smallest and the largest scale, met by ones times the other: the sums are ordinary numbers.  By bf16 instructions an element counts
    as a bf16 number."""
    q = np.zeros((m, 128), np.uint8)
    q[:, 0] = np.linspace(0, 126, m)
    one = np.zeros((3, 128), np.uint8)
    one[:, 0] = 0x38                                           # 1
    for low, high in ((1, 254), (254, 1)):
        a = put(q, np.full((m, 4), low, np.uint8), R.E4M3)
        b = put(one, np.full((3, 4), high, np.uint8), R.E4M3)
        c = torch.empty(m, 3, dtype=DT[kind], device="cuda")
        product(a, b, c, False, fp32_sums)
        want = np.repeat(R.decode(q[:, :1], R.E4M3), 3, 1)
        bound = np.zeros_like(want)
        if kind == "f32" or fp32_sums:
            if low == 1:
                bound = np.where(want < 2.0 ** -4, 2.0 ** -133 * 2.0 ** 126, 0)
            else:
                want = np.where(want >= 2, np.inf, want)
        got = c.double().cpu().numpy() / 2                     # 2^-126 times 2^127
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine], want[~fine]) and (np.abs(got[fine] - want[fine]) <= bound[fine]).all()
