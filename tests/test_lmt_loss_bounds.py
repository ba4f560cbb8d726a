"""The bounds that the GPU tests of the loss use, on a loss computed with fp32 roundings in numpy: they admit it, and find mistakes planted in it."""
import numpy as np
import pytest

from test_gpu_lmt_loss_accuracy import confident, formulas, loss_bound, sum_bound

F = np.float32


def in_fp32(x, t, w, cancel=False, sum_off=0.0):
    """Loss and gradient of one row, 256 lanes."""
    top = x.max()
    term = np.exp2(((x - top) * F(1.44269504088896340736)).astype(np.float64)).astype(F)
    lanes = np.zeros(256, F)
    for i in range(0, len(term), 256):
        part = term[i:i + 256]
        lanes[:len(part)] += part
    while len(lanes) > 1:
        lanes = lanes[::2] + lanes[1::2]
    total = F(lanes[0] * F(1 + sum_off))
    log = F(np.log(float(total)))
    loss = F(w) * (F(top + log) - x[t] if cancel else F(F(top - x[t]) + log))
    return float(loss), term * F(F(w) / total)


def misses(gap, offset, **mistake):
    rng = np.random.default_rng(7)
    x, t, w = confident(rng, 20, 5000, gap, offset)
    x = x.astype(F)
    loss, p, d, log_sum = formulas(x, t, w)
    rel = sum_bound(p, d, 5000)
    got = [in_fp32(x[i], t[i], w[i], **mistake) for i in range(20)]
    off = np.abs(np.array([l for l, _ in got]) - loss) > loss_bound(loss, p, d, log_sum, t, w, 5000)
    others = np.arange(5000)[None, :] != t[:, None]
    far = np.abs(np.array([g for _, g in got], np.float64) - w[:, None] * p) > w[:, None] * p * ((3 * np.abs(d) + 8) * 2.0 ** -24 + rel[:, None])
    return int(off.sum()), int((far & others).sum())


@pytest.mark.parametrize("gap", [0, 5, 14])
@pytest.mark.parametrize("offset", [0, 60, 3000])
def test_fp32_roundings_are_within(gap, offset):
    assert misses(gap, offset) == (0, 0)


def test_a_loss_that_cancels_is_found():
    assert misses(14, 3000, cancel=True)[0] > 10


def test_a_sum_off_by_a_ten_thousandth_is_found():
    loss, grad = misses(5, 0, sum_off=1e-4)
    assert loss > 15 and grad > 50000
