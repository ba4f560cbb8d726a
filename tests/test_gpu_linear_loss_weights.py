"""The loss of x table^T with weights that lie far apart: every row keeps its own bits (GPU)."""
import numpy as np
import pytest
import torch

import attention_reference as A
from lmt_gpu import DT, typed, within
from paper_2402_02447_amd import lmt
from test_gpu_linear_loss import IGNORE, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("outputs", ["loss lse grad_x grad_table", "grad_x", "loss grad_table"])
@pytest.mark.parametrize("rows", [5, 200, 256, 257, 300])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_small_weights_beside_large_ones(kind, rows, outputs):
    """Weights from 0.1 to 10^7 over a table whose rows have a mean, so that a row's gradient is half the target's and half that of 4 000 classes with a
    probability of 2^-12 each; elements of the table of 10^-3, so that the gradients are within fp16's range."""
    rng = np.random.default_rng(rows)
    x, _, t, _ = make(rng, rows, 4000, 64, kind)
    table = typed(1e-3 * (1 + 0.3 * rng.normal(0, 1, (4000, 64))), kind)
    w = (10.0 ** rng.uniform(-1, 7, rows)).astype(np.float32)
    w[:2] = 0.1, 1e7
    check(x, table, t, w, kind, outputs=outputs, f32=True)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [7, 256, 257])
def test_weights_of_any_size_and_none(kind, rows):
    rng = np.random.default_rng(rows)
    x, table, t, w = make(rng, rows, 700, 72, kind)
    w[::3] = 0
    w[1::3] *= -1
    check(x, table, t, w * np.float32(2.0 ** 60), kind, outputs="loss lse grad_table", f32=True)
    check(x, table, t, w * np.float32(2.0 ** -100), kind, f32=True)
    w[::5] = 2.0 ** -140
    check(x, table, t, w, kind, f32=True, outputs="lse grad_x grad_table")
    # a loss below fp32's smallest normal number is a multiple of 2^-149, off by up to half of that, which the bound of its roundings does not count
    loss = torch.empty(rows, device="cuda")
    X, TABLE = (torch.tensor(a).to(DT[kind]).cuda() for a in (x, table))
    ws = torch.empty(lmt.linear_cross_entropy_workspace(rows, 700, 72, False), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    lmt.linear_cross_entropy(X, TABLE, torch.tensor(t).cuda(), ws, loss, weights=torch.tensor(w).cuda(), ignore=IGNORE)
    torch.cuda.synchronize()
    want, bound = A.linear_loss(x, table, t, w, IGNORE, kind)["loss"]
    within(loss.cpu().numpy(), want, bound + 2.0 ** -150)
    check(x, table, t, None, kind, f32=True, accumulate=True)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("rows,classes,width", [(100, 700, 64), (300, 3000, 192), (300, 900, 72), (4000, 50_000, 64)])
def test_a_workspace_of_exactly_the_calls_size(kind, rows, classes, width):
    """Nothing behind it is touched, and the bits are those of one that is enough for any call."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x, table = torch.randn(rows, width, generator=g, device="cuda").to(DT[kind]), (torch.randn(classes, width, generator=g, device="cuda") / 4).to(DT[kind])
    t, w = torch.randint(classes, (rows,), generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    results = []
    for n in (lmt.linear_cross_entropy_workspace(rows, classes, width, dtype=DT[kind]), lmt.linear_cross_entropy_workspace(rows, classes, width)):
        buffer = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        out = [torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros_like(x), torch.zeros_like(table)]
        torch.cuda.synchronize()
        lmt.linear_cross_entropy(x, table, t, buffer[:n], *out, weights=w)
        torch.cuda.synchronize()
        assert bool((buffer[n:] == 0x5A).all())
        results.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*results))
