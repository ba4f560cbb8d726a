"""What rows of other sequences, and of none, hold is no concern of attention's gradients: infinities, large numbers and rows of unlike sizes beside
each other in one wavefront's 32 (GPU)."""
import math

import numpy as np
import pytest
import torch

import attention_reference as A
from lmt_gpu import DT, typed, within
from lmt_reference import TINY, U32, UNIT
from paper_2402_02447_amd import lmt
from test_gpu_attention import check

pytestmark = pytest.mark.gpu


def table(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def calls(q, k, v, go, starts, causal=False, **masks):
    """out, lse and the gradients of q, k and v."""
    T, H, D = q.shape
    starts = table(starts)
    out, lse = torch.full_like(q, 7.0), torch.full((H, T), 7.0, device="cuda")
    grads = [torch.full_like(x, 7.0) for x in (q, k, v)]
    ws = torch.full((lmt.attention_grad_workspace(T, H, k.shape[1], D),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    lmt.attention(q, k, v, out, lse, starts, causal=causal, **masks)
    lmt.attention_grad(go, q, k, v, out, lse, *grads, ws, starts, causal=causal, **masks)
    torch.cuda.synchronize()
    return out, lse, *grads


@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("masks", [dict(), dict(causal=True), dict(cap=4.0)], ids=str)
@pytest.mark.parametrize("first", [40, 2300, 3000])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_an_infinite_gradient_stays_in_its_sequence(kind, first, masks, size):
    """The last row of a long sequence has it; the next one begins in the same 32 rows.  Its gradients are what they are without the first one."""
    rng = np.random.default_rng(first)
    T = first + 70
    q, k, v, go = (typed(rng.normal(0, s, (T, 1, size)), kind) for s in (1.0, 1.0, 1.0, 0.01))
    go[first - 1, 0, 3] = np.inf
    on = [torch.tensor(x).to(DT[kind]).cuda() for x in (q, k, v, go)]
    masks = dict(masks, scale=1 / math.sqrt(size))
    out, lse, *got = calls(*on, [0, first, T], **masks)
    rest = slice(first, T)
    want = A.attention_grad(*(x[rest] for x in (go, q, k, v)), out.double().cpu().numpy()[rest], lse.double().cpu().numpy()[:, rest], [0, 70], kind, **masks)
    for x, (w, b) in zip(got, want):
        within(x.double().cpu().numpy()[rest], w, b)
    assert not bool(torch.isfinite(got[0][first - 1]).all()) and bool(torch.isfinite(got[0][:first - 1]).all())


def held(sigma, rows):
    """Puts numbers of this size, or what is no number, into the rows that nobody sees."""
    def spoil(q, k, v, go):
        rng = np.random.default_rng(5)
        for x in (q, k, v, go):
            for r in rows:
                n = x[r].shape
                x[r] = sigma if not np.isfinite(sigma) else np.clip(typed(typed(rng.normal(0, sigma, n), "bf16"), "f16"), -65280, 65280)     # of either type
    return spoil


@pytest.mark.parametrize("size", [64, 72, 128])
@pytest.mark.parametrize("general", [dict(), dict(cap=40.0, slopes=[0.01, -0.02])], ids=["plain", "general"])
@pytest.mark.parametrize("sigma", [8.0, 12.0, 100.0, 6e4, math.inf, math.nan])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_padding_beside_live_rows_may_hold_anything(kind, sigma, general, size):
    """300 live rows in 512: the last 12 share a wavefront with padding, while whole tiles lie inside of what they see."""
    rows = [slice(300, 512), slice(812, 1024)]
    check([0, 512, 1024], size=size, kind=kind, rows=1024, lengths=[300, 300], spoil=held(sigma, rows), **general)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("sigma", [12.0, math.inf])
def test_padding_beside_live_rows_that_have_no_gradient(kind, sigma):
    def spoil(q, k, v, go):
        held(sigma, [slice(300, 512)])(q, k, v, go)
        go[:300] = 0
    got = check([0, 512], size=64, kind=kind, rows=512, lengths=[300], spoil=spoil)[2:]
    assert not any(bool(x.view.any()) for x in got)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [300, 321, 1100])
def test_scores_that_rise_with_the_distance(kind, rows):
    """Lanes behind the last row work on that row's numbers, further away."""
    check([0, rows], heads=2, kv_heads=1, size=64, kind=kind, slopes=[-3.0, 0.05])
    check([0, rows - 70, rows], heads=2, kv_heads=1, size=32, kind=kind, slopes=[-1.0, -0.5])


def in_64_bits(go, q, k, v, out, lse, causal, scale, kind):
    """Gradients of one sequence on the GPU and their bounds: roundings of p and d to `kind` (an fp16 one as far below the largest of its row, of q or k, as 2^-38), of
    scores, exponentials and sums in fp32 as attention_reference.py counts them, of the result."""
    T, H, D = q.shape
    G = k.shape[1]
    unit, floor = UNIT[kind], 2.0 ** -38 if kind == "f16" else 0.0
    grads = [torch.zeros(T, n, D, dtype=torch.float64, device="cuda") for n in (H, G, G)]
    bounds = [torch.zeros_like(x) for x in grads]
    i = torch.arange(T, device="cuda")
    hidden = i[None, :] > i[:, None] if causal else None
    largest = torch.zeros(G, T, dtype=torch.float64, device="cuda")     # of a key's d, over all query heads that use it
    later = []

    def mm(a, b):
        return a @ b.contiguous()
    for h in range(H):
        g = h * G // H
        Q, K, V, GO, O = (x.double() for x in (q[:, h], k[:, g], v[:, g], go[:, h], out[:, h]))
        s, size = mm(Q, K.t()) * scale, mm(Q.abs(), K.abs().t()) * scale
        L = lse[h].double()[:, None]
        p = torch.exp(s - L)
        if causal:
            p = p.masked_fill(hidden, 0.0)
        rel = U32 * (D + 4) * size + 3 * U32 * s.abs() + U32 * (6 + 4 * L.abs())
        delta = (GO * O).sum(1, keepdim=True)
        e_dp = U32 * (D + 3) * (mm(GO.abs(), V.abs().t()) + (GO * O).abs().sum(1, keepdim=True))
        d = p * (mm(GO, V.t()) - delta)
        e_d = d.abs() * (rel + 6 * U32) + p * e_dp
        sums = (T * H // G + 4) * U32
        rough = e_d + unit * (d.abs() + e_d) + sums * d.abs()
        low = floor * (d.abs() + e_d).amax(1, keepdim=True) * (p > 0)
        grads[0][:, h] += scale * mm(d, K)
        bounds[0][:, h] += scale * mm(rough + low, K.abs())
        grads[1][:, g] += scale * mm(d.t(), Q)
        bounds[1][:, g] += scale * mm(rough.t(), Q.abs())
        largest[g] = torch.maximum(largest[g], (d.abs() + e_d).amax(0))
        later.append((g, mm((p > 0).double().t(), Q.abs())))
        grads[2][:, g] += mm(p.t(), GO)
        bounds[2][:, g] += mm((p * (rel + unit + sums) + floor * (p > 0)).t(), GO.abs())
    for g, x in later:
        bounds[1][:, g] += scale * floor * largest[g][:, None] * x
    return [(x, 1.01 * (b + unit * x.abs()) + TINY[kind] + 2.0 ** -100) for x, b in zip(grads, bounds)]


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("T,heads,kv_heads,size,causal", [(3000, 8, 1, 128, True), (2500, 8, 2, 128, False), (1000, 4, 4, 64, True), (515, 16, 1, 64, False)])
def test_rows_of_unlike_sizes(kind, T, heads, kv_heads, size, causal):
    """Long sequences, parts of the query heads, and gradients whose rows differ by up to 2^20: every row keeps its own bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    q, go = (torch.randn(T, heads, size, generator=g, device="cuda") for _ in range(2))
    k, v = (torch.randn(T, kv_heads, size, generator=g, device="cuda") for _ in range(2))
    go *= 2.0 ** -(20 * torch.rand(T, 1, 1, generator=g, device="cuda"))
    v *= 2.0 ** -(10 * torch.rand(T, 1, 1, generator=g, device="cuda"))
    q, k, v, go = (x.to(DT[kind]) for x in (q, k, v, go))
    scale = 2.0 / math.sqrt(size)
    out, lse, *got = calls(q, k, v, go, [0, T], causal, scale=scale)
    for x, (w, b) in zip(got, in_64_bits(go, q, k, v, out, lse, causal, scale, kind)):
        over = (x.double() - w).abs() - b
        assert bool(torch.isfinite(x).all()) and float(over.max()) <= 0, (int((over > 0).sum()), float(over.max()))


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("T,heads,kv_heads,size,causal", [(3000, 8, 1, 128, True), (4100, 2, 2, 128, False), (2500, 4, 2, 64, True), (1777, 3, 3, 96, False)])
def test_results_of_long_sequences(kind, T, heads, kv_heads, size, causal):
    """Scores spread over some 2^20, so that the running largest of a row moves many times.  Bounds as attention_reference.py counts them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    q = torch.randn(T, heads, size, generator=g, device="cuda").to(DT[kind])
    k, v = (torch.randn(T, kv_heads, size, generator=g, device="cuda").to(DT[kind]) for _ in range(2))
    scale, unit = 4.0 / math.sqrt(size), UNIT[kind]
    out, lse = torch.full_like(q, 7.0), torch.full((heads, T), 7.0, device="cuda")
    torch.cuda.synchronize()
    lmt.attention(q, k, v, out, lse, table([0, T]), scale=scale, causal=causal)
    torch.cuda.synchronize()
    i = torch.arange(T, device="cuda")
    hidden = (i[None, :] > i[:, None]) & causal
    for h in range(heads):
        Q, K, V = (x.double() for x in (q[:, h], k[:, h * kv_heads // heads], v[:, h * kv_heads // heads]))
        s, off = Q @ K.t().contiguous() * scale, Q.abs() @ K.abs().t().contiguous() * scale * (U32 * (size + 4))
        off = (off + 3 * U32 * s.abs()).masked_fill(hidden, 0.0)
        s = s.masked_fill(hidden, -math.inf)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        p /= total
        worst = off.amax(1, keepdim=True) + U32 * (i[:, None] * causal + T * (not causal) + 9 + 4 * top.abs())
        want, size_of = p @ V, p @ V.abs()
        low = (~hidden).double() @ V.abs()
        bound = 1.01 * (size_of * (unit + 2 * worst) + 2.0 ** -31 * low * (kind == "f16") + unit * want.abs() + TINY[kind] + 2.0 ** -126 * (low + T))
        want_lse = (top + torch.log(total)).squeeze(1)
        assert float(((out[:, h].double() - want).abs() - bound).max()) <= 0
        assert float(((lse[h].double() - want_lse).abs() - 1.01 * (worst.squeeze(1) + 4 * U32 * want_lse.abs()) - 2 * U32).max()) <= 0
