"""The loss of x table^T and its gradients against their formulas in 64 bits (GPU)."""
import numpy as np
import pytest
import torch

import attention_reference as A
from lmt_gpu import DT, Mat, typed, within
from paper_2402_02447_amd import lmt

pytestmark = pytest.mark.gpu
IGNORE = -100


def make(rng, n, V, W, kind, sigma=2.0):
    x, table = typed(rng.normal(0, 1, (n, W)), kind), typed(rng.normal(0, sigma / np.sqrt(W), (V, W)), kind)
    t = rng.integers(0, V, n)
    t[rng.random(n) < 0.2] = IGNORE
    return x, table, t, rng.uniform(0.1, 2, n).astype(np.float32)


def check(x, table, t, w, kind="bf16", ids="i64", gap=0, offset=0, ignore=IGNORE, outputs="loss lse grad_x grad_table", f32=False, accumulate=False, status=0, stream=None):
    n, W = x.shape
    V = table.shape[0]
    X, TABLE = Mat(n, W, kind, gap, offset, x), Mat(V, W, kind, gap, offset, table)
    kt = "f32" if f32 else kind
    old = typed(np.random.default_rng(9).normal(0, 0.1, (V, W)), kt) if accumulate else None
    GX, GT = Mat(n, W, kind, gap + 1, offset), Mat(V, W, kt, gap + 2, offset + 1, old)
    T = torch.as_tensor(np.asarray(t, np.int64)).to(DT[ids]).cuda()
    Wt = None if w is None else torch.tensor(w, dtype=torch.float32, device="cuda")
    loss, lse = (torch.full((n,), 77.0, device="cuda") if o in outputs.split() else None for o in ("loss", "lse"))
    there = torch.zeros(1, dtype=torch.int32, device="cuda")
    grads = "grad" in outputs
    ws = torch.full((lmt.linear_cross_entropy_workspace(n, V, W, grads),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    lmt.linear_cross_entropy(X.view, TABLE.view, T, ws, loss, lse, GX.view if "grad_x" in outputs else None, GT.view if "grad_table" in outputs else None, Wt, ignore, accumulate, there, stream)
    torch.cuda.synchronize()
    want = A.linear_loss(x, table, np.asarray(t), w, ignore, kind, kt, old)
    for name, got in (("loss", loss), ("lse", lse), ("grad_x", GX), ("grad_table", GT)):
        if name in outputs.split():
            within(got.numpy() if isinstance(got, Mat) else got.cpu().numpy(), *want[name])
    assert X.untouched_outside() and TABLE.untouched_outside() and GX.untouched_outside() and GT.untouched_outside()
    assert np.array_equal(X.numpy(), x, equal_nan=True) and int(there.item()) == status


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,V,W", [(1, 1, 1), (1, 2, 3), (2, 5, 64), (63, 65, 7), (64, 64, 64), (65, 63, 65), (127, 129, 128), (128, 128, 100), (129, 256, 33), (300, 257, 192), (5, 3000, 200),
                                   (700, 40, 96), (257, 1000, 257), (40, 9000, 64), (3000, 130, 40)])
def test_sizes(kind, n, V, W):
    rng = np.random.default_rng(n + V + W)
    x, table, t, w = make(rng, n, V, W, kind)
    check(x, table, t, w, kind)
    check(x, table, t, None, kind, "i32", gap=3, offset=1, accumulate=True)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("accumulate", [False, True])
def test_types_of_the_tables_gradient(kind, f32, accumulate):
    x, table, t, w = make(np.random.default_rng(1), 150, 500, 128, kind)
    check(x, table, t, w, kind, f32=f32, accumulate=accumulate)
    check(x, table, t, w / 1e6, kind, f32=f32, accumulate=accumulate)          # weights of a mean: fp16's range is no concern of theirs


@pytest.mark.parametrize("outputs", ["loss", "lse", "grad_x", "grad_table", "loss grad_table", "lse grad_x", ""])
def test_any_output_may_be_left_out(outputs):
    x, table, t, w = make(np.random.default_rng(2), 90, 300, 64, "bf16")
    check(x, table, t, w, outputs=outputs)


@pytest.mark.parametrize("sigma", [0.0, 0.01, 30.0, 300.0])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_flat_and_peaked_rows(sigma, kind):
    x, table, t, w = make(np.random.default_rng(3), 70, 400, 64, kind, sigma)
    t[:30] = (x @ table.T)[:30].argmax(1)
    check(x, table, t, w, kind)


def test_ignored_rows_take_no_part_whatever_they_hold():
    x, table, t, w = make(np.random.default_rng(4), 200, 300, 96, "bf16")
    t[:] = np.where(t == IGNORE, 5, t)
    clean = x.copy()
    t[[3, 64, 130, 199]] = IGNORE
    x[3], x[64], x[130] = np.nan, np.inf, -np.inf
    w[199] = np.nan
    clean[[3, 64, 130]] = 0
    X, TABLE = Mat(200, 96, "bf16", values=x), Mat(300, 96, "bf16", values=table)
    GX, GT = Mat(200, 96, "bf16"), Mat(300, 96, "bf16")
    loss = torch.full((200,), 7.0, device="cuda")
    ws = torch.empty(lmt.linear_cross_entropy_workspace(200, 300, 96), dtype=torch.uint8, device="cuda")
    lmt.linear_cross_entropy(X.view, TABLE.view, torch.tensor(t).cuda(), ws, loss, None, GX.view, GT.view, torch.tensor(w).cuda())
    torch.cuda.synchronize()
    w[199] = 1
    want = A.linear_loss(clean, table, t, w, IGNORE, "bf16")
    within(loss.cpu().numpy(), *want["loss"])
    within(GX.numpy(), *want["grad_x"])
    within(GT.numpy(), *want["grad_table"])


def test_targets_that_are_none():
    x, table, t, w = make(np.random.default_rng(5), 60, 50, 32, "bf16")
    t[:5] = [50, -1, 2 ** 31 - 1, -2 ** 31, 51]
    check(x, table, t, w, ids="i32", status=lmt.LMT_STATUS_BAD_TARGET)
    t[:3] = [2 ** 40 + 3, -2 ** 63, 2 ** 32 + 7]
    check(x, table, t, w, status=lmt.LMT_STATUS_BAD_TARGET)
    t[:] = 7
    check(x, table, t, w, ignore=7)
    t[:] = np.random.default_rng(1).integers(0, 50, 60)
    check(x, table, t, np.zeros(60, np.float32))
    check(x, table, t, -w)


def test_nan_of_a_row_stays_in_its_results_and_the_tables_gradient():
    x, table, t, w = make(np.random.default_rng(6), 140, 300, 64, "bf16")
    t[70] = 4
    x[70] = np.nan
    X, TABLE, GX = Mat(140, 64, "bf16", values=x), Mat(300, 64, "bf16", values=table), Mat(140, 64, "bf16")
    loss, lse = (torch.zeros(140, device="cuda") for _ in range(2))
    ws = torch.empty(lmt.linear_cross_entropy_workspace(140, 300, 64), dtype=torch.uint8, device="cuda")
    lmt.linear_cross_entropy(X.view, TABLE.view, torch.tensor(t).cuda(), ws, loss, lse, GX.view, None, torch.tensor(w).cuda())
    torch.cuda.synchronize()
    bad = np.zeros(140, bool)
    bad[70] = True
    for got in (loss, lse, GX.view[:, 0]):
        assert np.array_equal(~torch.isfinite(got.float()).cpu().numpy(), bad)


def test_pieces_of_the_classes():
    """More classes than one piece has (2^27 elements of the gradient at 3 000 rows and 100 000 classes), against the same rows in 64 bits on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n, V, W = 3000, 100_001, 64
    x, table = torch.randn(n, W, generator=g, device="cuda").bfloat16(), (torch.randn(V, W, generator=g, device="cuda") / 4).bfloat16()
    t = torch.randint(V, (n,), generator=g, device="cuda")
    t[-40:] = torch.arange(V - 40, V, device="cuda")
    loss, lse, gx, gt = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty_like(table)
    ws = torch.empty(lmt.linear_cross_entropy_workspace(n, V, W), dtype=torch.uint8, device="cuda")
    lmt.linear_cross_entropy(x, table, t, ws, loss, lse, gx, gt)
    torch.cuda.synchronize()
    logits = x.double() @ table.double().t()
    total = torch.logsumexp(logits, 1)
    # W + V roundings of sums at most, far fewer in fact: 1e-6 of a logit's size (30) and of the sum
    assert float((lse - total).abs().max()) <= 3e-5 and float((loss - (total - logits.gather(1, t[:, None]).squeeze(1))).abs().max()) <= 6e-5
    d = torch.exp(logits - total[:, None])
    d[torch.arange(n), t] -= 1
    # two roundings of half a step (2^-9 of a value on average below 2^-8) in the 2-norm
    for got, want in ((gx, d @ table.double()), (gt, d.t().contiguous() @ x.double())):
        assert float((got.double() - want).norm() / want.norm()) <= 2.0 ** -8
        assert float((got.double() - want)[-1000:].norm() / want[-1000:].norm()) <= 2.0 ** -8


def test_the_same_call_gives_the_same_bits_and_a_graph_follows_its_inputs():
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    n, V, W = 500, 2000, 128
    x, table = torch.randn(n, W, generator=g, device="cuda").half(), torch.randn(V, W, generator=g, device="cuda").half() / 8
    t = torch.zeros(n, dtype=torch.int64, device="cuda")

    def state():
        return [torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros_like(x), torch.zeros_like(table), torch.empty(lmt.linear_cross_entropy_workspace(n, V, W), dtype=torch.uint8, device="cuda")]

    def step(s, stream=None):
        lmt.linear_cross_entropy(x, table, t, s[4], *s[:4], stream=stream)
    a, b, c = state(), state(), state()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step(b, stream)
    for _ in range(4):
        t.copy_(torch.randint(V, (n,), generator=g, device="cuda"))
        x.copy_(torch.randn(n, W, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        step(a)
        torch.cuda.synchronize()
        step(c)
        torch.cuda.synchronize()
        for p, q, r in zip(a[:4], b[:4], c[:4]):
            assert torch.equal(p, q) and torch.equal(p, r)
