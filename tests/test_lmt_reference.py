"""The 64-bit reference of the operators of lmt.h, held to independent statements of the same things."""
import numpy as np
import pytest
import torch

import lmt_reference as R


@pytest.mark.parametrize("form,dtype", [(R.E4M3, torch.float8_e4m3fn), (R.E5M2, torch.float8_e5m2)])
def test_codes_stand_for_the_types_values(form, dtype):
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(dtype).double().numpy()
    assert np.array_equal(R.decode(codes, form), want, equal_nan=True)
    assert np.nanmax(np.where(np.isfinite(want), want, np.nan)) == R.LARGEST[form]


@pytest.mark.parametrize("form,dtype", [(R.E4M3, torch.float8_e4m3fn), (R.E5M2, torch.float8_e5m2)])
def test_rounding_is_to_the_nearest_value_with_ties_to_even(form, dtype):
    v = R.decode(np.arange(127 if form == R.E4M3 else 124), form)
    mid = (v[1:] + v[:-1]) / 2
    y = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), np.random.default_rng(0).normal(0, 50, 1000)])
    y = np.concatenate([y, -y])
    y32 = y.astype(np.float32)
    y32 = y32[np.abs(y32) <= R.LARGEST[form]]
    got = R._encode(y32.astype(np.float64), form)
    assert np.array_equal(got, torch.from_numpy(y32).to(dtype).view(torch.uint8).numpy())


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("form", [R.E4M3, R.E5M2])
def test_scales_are_the_smallest_that_are_enough(form, tile):
    rng = np.random.default_rng(1)
    x = (rng.normal(0, 1, (130, 257)) * np.exp(rng.normal(0, 8, (130, 1)))).astype(np.float32)
    x[3, 128:256] = 0
    q, s = R.quantize(x, form, tile)
    assert q.shape == (130, 384) and s.shape == (130, 4)
    assert np.all(s[:, 3:] == 127) and np.all(q[:, 257:] & 127 == 0)
    v = R.values(q, s, form)[:, :257]
    for i in range(130):
        for b in range(3):
            rows = slice(i // 128 * 128, min(130, i // 128 * 128 + 128)) if tile else slice(i, i + 1)
            size = np.abs(x[rows, 128 * b:128 * b + 128].astype(np.float64)).max()
            scale = 2.0 ** (float(s[i, b]) - 127)
            assert size / scale <= R.LARGEST[form]
            assert s[i, b] == 1 or size / (scale / 2) > R.LARGEST[form]
    # the largest relative error of a value that is not below the type's normal range is half a unit of its mantissa
    big = np.abs(x) >= np.repeat(2.0 ** (s[:, :3].astype(np.float64) - 127), 128, 1)[:, :257] * 2.0 ** (-6 if form == R.E4M3 else -14)
    assert np.all(np.abs(v - x)[big] <= np.abs(x)[big] * 2.0 ** (-4 if form == R.E4M3 else -3))


def test_gradients_are_the_differences_of_what_they_belong_to():
    rng = np.random.default_rng(2)
    x, t, w = rng.normal(0, 2, (5, 11)), np.array([0, 10, -100, 4, 4]), rng.uniform(0.1, 1, 5)
    (_, _, grad), _ = R.cross_entropy(x, t, w, -100)
    h = 1e-6
    for i in range(5):
        for j in range(11):
            up, down = x.copy(), x.copy()
            up[i, j] += h
            down[i, j] -= h
            d = (R.cross_entropy(up, t, w, -100)[0][0].sum() - R.cross_entropy(down, t, w, -100)[0][0].sum()) / (2 * h)
            assert abs(d - grad[i, j]) <= 1e-8
    # sum over t, j of g[t][j] out[t][j] is linear in the table: its derivative is embed_grad
    tokens, table, g = np.array([3, 0, 3, 1, 3, 0]), rng.normal(0, 1, (4, 3)), rng.normal(0, 1, (6, 3))
    grad, _ = R.embed_grad(g, tokens, 4, 0.7, 0)
    for v in range(4):
        for j in range(3):
            up, down = table.copy(), table.copy()
            up[v, j] += h
            down[v, j] -= h
            d = ((R.embed(up, tokens, 0.7) - R.embed(down, tokens, 0.7)) * g).sum() / (2 * h)
            assert abs(d * (v != 0) - grad[v, j]) <= 1e-8


def test_empty_rows_and_values_that_are_none():
    inf, nan = np.inf, np.nan
    x = np.array([[-inf, -inf, -inf], [-inf, 0, 0], [inf, 0, 0], [nan, 0, 0], [nan, -inf, -inf]])
    (loss, lse, grad), _ = R.cross_entropy(x, np.array([0, 0, 0, 0, 0]), None, -100)
    assert lse[0] == -inf and loss[0] == inf and not grad[0].any()
    assert lse[1] == np.log(2) and loss[1] == inf and np.array_equal(grad[1], [-1, 0.5, 0.5])
    assert np.isnan(lse[2:]).all() and np.isnan(loss[2:]).all() and np.isnan(grad[2:]).all()
    (loss, lse, grad), _ = R.cross_entropy(x, np.full(5, -100), None, -100)
    assert not loss.any() and not grad.any()
