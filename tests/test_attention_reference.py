"""The formulas of attention_reference.py against differences and against each other, without a GPU."""
import numpy as np
import pytest

import attention_reference as A

CASES = [dict(), dict(causal=True), dict(causal=True, prefixes=[2, 0, 9]), dict(slopes=[0.3, 0.02, 0.0, 1.0]), dict(cap=1.5), dict(cap=0.7, slopes=[0.1, 0.2, 0.3, 0.4], causal=True), dict(scale=-0.4)]


def inputs(seed=0, T=14, H=4, G=2, D=3):
    r = np.random.default_rng(seed)
    return r.normal(size=(T, H, D)), r.normal(size=(T, G, D)), r.normal(size=(T, G, D)), r.normal(size=(T, H, D)), [1, 5, 5, 11], [4, 0, 6]


@pytest.mark.parametrize("masks", CASES, ids=str)
def test_gradients_of_attention_are_differences_of_its_results(masks):
    q, k, v, go, starts, lengths = inputs()
    masks = dict(dict(scale=0.6), **masks)

    def total(*x):
        return float((A.attention(*x, starts, "bf16", lengths, **masks)[0][0] * go).sum())
    (out, _), (lse, _) = A.attention(q, k, v, starts, "bf16", lengths, **masks)
    grads = A.attention_grad(go, q, k, v, out, lse, starts, "bf16", lengths, **masks)
    step = 1e-5
    for n, x in enumerate((q, k, v)):
        for at in np.ndindex(*x.shape):
            x[at] += step
            up = total(q, k, v)
            x[at] -= 2 * step
            down = total(q, k, v)
            x[at] += step
            assert abs((up - down) / (2 * step) - grads[n][0][at]) <= 1e-8, (n, at)   # step^2 and 2^-53 / step, both about 1e-10


def test_gradients_of_the_loss_are_differences():
    r = np.random.default_rng(1)
    x, table, w = r.normal(size=(5, 4)), r.normal(size=(7, 4)), r.uniform(0.5, 2, 5)
    t = np.array([3, -100, 0, 6, 9])
    got = A.linear_loss(x, table, t, w, -100, "bf16")
    for name, a in (("grad_x", x), ("grad_table", table)):
        for at in np.ndindex(*a.shape):
            a[at] += 1e-5
            up = A.linear_loss(x, table, t, w, -100, "bf16")["loss"][0].sum()
            a[at] -= 2e-5
            down = A.linear_loss(x, table, t, w, -100, "bf16")["loss"][0].sum()
            a[at] += 1e-5
            assert abs((up - down) / 2e-5 - got[name][0][at]) <= 1e-8


def test_rotary_turns_pairs_and_back():
    r = np.random.default_rng(2)
    x, pos, f = r.normal(size=(6, 2, 11)), r.integers(-5, 2000, 6), r.uniform(0.01, 1, 4)
    for neighbours in (False, True):
        y = A.rotary(x, pos, f, 1.0, neighbours)[0]
        z = A.rotary(y, pos, f, 1.0, neighbours, True)[0]
        assert np.allclose(z, x, atol=1e-12) and np.array_equal(y[..., 8:], x[..., 8:])
        a, b = (x[..., 0:8:2], x[..., 1:8:2]) if neighbours else (x[..., :4], x[..., 4:8])
        c, d = (y[..., 0:8:2], y[..., 1:8:2]) if neighbours else (y[..., :4], y[..., 4:8])
        turned = (a + 1j * b) * np.exp(1j * pos[:, None, None] * f)
        assert np.allclose(c + 1j * d, turned, atol=1e-12)


def test_planted_mistakes_leave_the_bounds():
    """A causal mask off by one, a forgotten slope, a derivative without the cap, a head's gradient left out of a shared one."""
    q, k, v, go, starts, lengths = inputs(3, T=40, D=8)
    starts, lengths = [0, 20, 20, 38], [20, 0, 15]
    right = dict(scale=0.5, cap=2.0, slopes=[0.05, 0.1, 0.2, 0.4], causal=True)
    (out, b), (lse, b_lse) = A.attention(q, k, v, starts, "bf16", lengths, **right)
    for wrong in (dict(causal=False), dict(slopes=None), dict(cap=0.0), dict(prefixes=[3, 0, 0])):
        (o, _), (s, _) = A.attention(q, k, v, starts, "bf16", lengths, **dict(right, **wrong))
        assert (np.abs(o - out) > b).any() and (np.abs(s - lse)[np.isfinite(lse)] > b_lse[np.isfinite(lse)]).any()
    grads = A.attention_grad(go, q, k, v, out, lse, starts, "bf16", lengths, **right)
    flat = A.attention_grad(go, q, k, v, out, lse, starts, "bf16", lengths, **dict(right, cap=0.0))
    assert (np.abs(flat[0][0] - grads[0][0]) > grads[0][1]).any()
    fewer = go.copy()
    fewer[:, 1] = 0
    less = A.attention_grad(fewer, q, k, v, out, lse, starts, "bf16", lengths, **right)
    assert all((np.abs(less[n][0] - grads[n][0]) > grads[n][1]).any() for n in (1, 2))
