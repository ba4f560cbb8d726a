"""How exact losses and their gradients are (GPU): bounds from the roundings that a subtraction of the maximum, exp2 and a sum over lanes take, with no part that grows
with the logits' common offset."""
import numpy as np
import pytest
import torch

from lmt_gpu import DT, Mat, typed, within
from lmt_reference import U32 as U, rounded
from paper_2402_02447_amd import lmt

pytestmark = pytest.mark.gpu


def formulas(x, t, w):
    """loss, probabilities, x - max and log of the sum of exp(x - max), in 64 bits.  x, t, w: numpy, every row counted and finite."""
    x, at = x.astype(np.float64), np.arange(len(x))
    d = x - x.max(1, keepdims=True)
    e = np.exp(d)
    # the target's term apart, so that a loss of a probability near 1 keeps its digits
    others = e.copy()
    others[at, t] = 0
    others = others.sum(1)
    loss = w * np.where(d[at, t] == 0, np.log1p(others), np.log(others + e[at, t]) - d[at, t])
    return loss, e / e.sum(1, keepdims=True), d, np.log(e.sum(1))


def sum_roundings(V):
    """Additions a term goes through: up to 128 of a lane's own, or its share of a longer row; 6 over a wavefront, 16 over a workgroup."""
    return max(128, -(-V // 1024) + 8) + 22


def sum_bound(p, d, V):
    """Relative error of a row's sum: of each term 3 |d| u (the difference, log2(e) and their product, each rounded) and 3 u of exp2; the additions."""
    return (p * (3 * np.abs(d) + 3)).sum(1) * U + sum_roundings(V) * U


def loss_bound(loss, p, d, log_sum, t, w, V):
    """The difference to the target, the sum, its logarithm (2 u of itself and 2 u near 0), their sum, the weight."""
    to_target = np.abs(d[np.arange(len(t)), t])
    return w * (U * to_target + sum_bound(p, d, V) + 2 * U * log_sum + 2 * U) + 2 * U * np.abs(loss)


def call(x, t, w, dtype, grad=False, lse=False):
    X = torch.as_tensor(x).to(DT[dtype]).cuda()
    loss = torch.empty(len(x), device="cuda")
    g = torch.empty_like(X) if grad else None
    s = torch.empty_like(loss) if lse else None
    lmt.cross_entropy(X, torch.as_tensor(t).cuda(), loss, s, g, torch.as_tensor(w, dtype=torch.float32).cuda())
    return [None if o is None else o.double().cpu().numpy() for o in (loss, s, g)]


def confident(rng, n, V, gap, offset):
    """The target is the largest logit, `gap` above a field of N(0, 1): losses of about V exp(1/2 - gap)."""
    x = rng.normal(0, 1, (n, V))
    t = rng.integers(0, V, n)
    x[np.arange(n), t] = gap
    return x + offset, t, np.float32(rng.uniform(0.5, 2, n)).astype(np.float64)


@pytest.mark.parametrize("V,gap", [(100, 12), (100, 18), (1000, 14), (30522, 18), (30522, 24), (200000, 20)])
@pytest.mark.parametrize("offset", [0, 20, 60, -300, 3000])
def test_a_small_loss_does_not_lose_to_the_logits_offset(V, gap, offset):
    x, t, w = confident(np.random.default_rng(V + gap), 40 if V < 1e5 else 6, V, gap, offset)
    x = typed(x, "f32")
    loss, p, d, log_sum = formulas(x, t, w)
    assert 1e-7 < loss.max() < 1e-1
    within(call(x, t, w, "f32")[0], loss, loss_bound(loss, p, d, log_sum, t, w, V))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [100, 3000, 30522, 200000])
def test_an_offset_of_every_logit_leaves_the_same_loss(dtype, V):
    """Logits of whole numbers and offsets that keep them so: x - max is the same bits, and so is all that follows."""
    rng = np.random.default_rng(V)
    x, t, w = rng.integers(-8, 9, (10, V)).astype(np.float64), rng.integers(0, V, 10), rng.uniform(0.5, 1, 10)
    t[:5] = x[:5].argmax(1)
    first = call(x, t, w, dtype, True)
    for offset in (-100, 64, 200) if dtype == "bf16" else (-1000, 64, 2000):
        near = call(x + offset, t, w, dtype, True)
        assert np.array_equal(typed(x + offset, dtype), x + offset)
        assert np.array_equal(first[0], near[0]) and np.array_equal(first[2], near[2])


@pytest.mark.parametrize("V", [200, 3000, 30522, 200000])
@pytest.mark.parametrize("width", [2, 4, 12])
def test_gradients_keep_the_low_bits_of_the_exponent(V, width):
    """y = (x - max) log2(e) by two fp32 operations, which numpy repeats; what remains of a gradient is 2^y times a factor of its row: an ulp, 2 u, for 2^y,
    u for the product, and as much for the median that stands for the factor.  (With an argument of 16 to 32 instead of y, errors reach 11 u more.)"""
    rng = np.random.default_rng(V)
    n = 12 if V < 1e5 else 4
    x = rng.uniform(-width, 0, (n, V)).astype(np.float32)
    grad = call(x, np.zeros(n, np.int64), np.ones(n), "f32", True)[2][:, 1:]      # the target has another formula
    y = ((x - x.max(1, keepdims=True)) * np.float32(1.44269504088896340736))[:, 1:]
    assert y.dtype == np.float32
    ratio = grad / np.exp2(y.astype(np.float64))
    assert (np.abs(ratio / np.median(ratio, 1, keepdims=True) - 1) <= 2 * (2 + 1) * U).all()


@pytest.mark.parametrize("V", [40, 3000, 200000])
def test_gradients_far_below_the_largest_are_not_cut_off(V):
    """Probabilities from 1 down to fp32's smallest, below which 0 is right."""
    rng = np.random.default_rng(V)
    x = typed(rng.uniform(-110, 0, (8 if V < 1e5 else 2, V)), "f32")
    x[:, 0] = 0
    t, w = np.ones(len(x), np.int64), np.ones(len(x))
    loss, p, d, log_sum = formulas(x, t, w)
    for scale in (1.0, 2.0 ** -20, 2.0 ** 20):
        grad = call(x, t, w * scale, "f32", True)[2]
        want = scale * p
        want[:, 1] -= scale
        bound = scale * p * (3 * np.abs(d) + 6 + sum_bound(p, d, V)[:, None] / U) * U + 2.0 ** -149
        bound[:, 1] += 2 * U * scale
        within(grad, want, bound)


SIZES = [(5, 1), (5, 2), (5, 7), (9, 8), (40, 255), (40, 257), (20, 1023), (10, 2049), (10, 4097), (6, 8193), (6, 16385), (4, 30522), (3, 32769), (3, 65537), (2, 131073), (2, 300001)]


@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("sigma,offset", [(2.0, 0.0), (0.01, 9.0), (20.0, -40.0)])
def test_every_output_within_the_roundings_of_sums_over_lanes(n, V, dtype, sigma, offset):
    """A relative 2e-5 at most at the usual sizes; what a gradient's own type rounds comes on top."""
    rng = np.random.default_rng(V)
    x = typed(rng.normal(offset, sigma, (n, V)), dtype)
    x[:, 1::7] = np.where(rng.random((n, 1)) < 0.5, -np.inf, x[:, 1::7])            # classes that cannot occur, in half of the rows
    x[n - 1, 0] = x[n - 1].max()                                                     # a tie, for the first place too
    t = np.where(rng.random(n) < 0.5, x.argmax(1), 0)
    w = np.float32(rng.uniform(0.1, 2, n)).astype(np.float64)
    loss, p, d, log_sum = formulas(x, t, w)
    d = np.where(p > 0, d, 0)
    rel = sum_bound(p, d, V)
    assert V > 1e5 or sigma > 2 or rel.max() < 2e-5
    at = np.arange(n)
    grad = w[:, None] * p
    # a gradient: what a term has, but 6 u of exp2 (its root twice, and their products), the quotient and its product 2; of the target's, the difference
    bound = grad * (3 * np.abs(d) + 8 + rel[:, None] / U) * U
    grad[at, t] = np.where(V > 1, w * (p[at, t] - 1), 0)
    bound[at, t] += 2 * U * w
    lse = x.max(1) + log_sum
    for in_place in (False, True):
        m = Mat(n, V, dtype, 3, 1, x)
        g = m if in_place else Mat(n, V, dtype, 2, 0)
        out, s = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        lmt.cross_entropy(m.view, torch.as_tensor(t).cuda(), out, s, g.view, torch.as_tensor(w, dtype=torch.float32).cuda())
        within(out.cpu().numpy(), loss, loss_bound(loss, p, d, log_sum, t, w, V))
        within(s.cpu().numpy(), lse, rel + 2 * U * log_sum + 2 * U + U * np.abs(lse))
        within(g.numpy(), grad, bound + rounded(np.abs(grad) + bound, dtype))
        assert g.untouched_outside() and m.untouched_outside()
