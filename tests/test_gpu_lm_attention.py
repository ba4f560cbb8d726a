"""A step of a model with an attention layer over sequences of unlike lengths, and with a loss that keeps no logits (GPU)."""
import math

import pytest
import torch

from paper_2402_02447_amd import lmt
from paper_2402_02447_amd.lm_step import IGNORE, PADDING, TiedLm, batch, sequences

pytestmark = pytest.mark.gpu


def turned(x, positions, inverse=False):
    half = x.shape[-1] // 2
    z = positions.double()[:, None, None] * lmt.rotary_frequencies(half).double().cuda()
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * z.cos() - b * z.sin(), a * z.sin() + b * z.cos()], 2)


def by_autograd(model, tokens, targets, weights, starts, positions):
    """Loss and gradients in 64 bits, from the formulas, without any operand in 8 or 16 bits."""
    params = [t.double().requires_grad_() for t in (model.table, model.proj) + ((model.qkv,) if model.heads else ())]
    table, proj = params[:2]
    x = table[tokens.long()] * model.scale
    x = torch.where((tokens == PADDING).unsqueeze(1), x.detach(), x)
    if model.heads:
        n, T = model.heads, x.shape[0]
        q, k, v = (x @ params[2].t()).view(T, 3, n, -1).unbind(1)
        q, k = turned(q, positions), turned(k, positions)
        at = torch.arange(T, device="cuda")
        of = torch.searchsorted(starts.long(), at, right=True)
        sees = (of[:, None] == of[None]) & (at[None] <= at[:, None])
        scores = torch.einsum("ihd,jhd->hij", q, k) * model.attend_scale
        p = torch.softmax(scores.masked_fill(~sees, -math.inf), 2)
        h = x + torch.einsum("hij,jhd->ihd", p, v).reshape(T, -1) @ proj.t()
    else:
        h = x @ proj.t()
    loss = (torch.nn.functional.cross_entropy(h @ table.t(), targets, ignore_index=IGNORE, reduction="none") * weights.double()).sum()
    return float(loss.detach()), torch.autograd.grad(loss, params)


def inputs(vocab, tokens, seed, longest=70):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return batch(vocab, tokens, g), sequences(tokens, longest, g)


@pytest.mark.parametrize("heads,logits", [(4, True), (4, False), (0, False)])
def test_gradients_of_a_step_are_those_of_the_formulas_up_to_the_operands_rounding(heads, logits):
    """Every 8-bit product rounds its operands to 3 mantissa bits (0.026 of a value on average over a binade) or, gradients, 2 (0.052), a relative error in the
    2-norm of 0.058; errors of unlike elements are independent.  With attention the weights' gradients go through at most five such products behind
    the loss (of h, the mix, the parts, their weights), whose logits come out of three in front of it: sqrt(8) 0.058 = 0.17.  Attention's own
    roundings to bf16 (2^-9 on average) are far below.  A loss that keeps no logits does with two products fewer."""
    model = TiedLm(vocab=777, width=256, tokens=1001, heads=heads, logits=logits)
    (tokens, targets, weights), (starts, positions) = inputs(777, 1001, 3)
    model.gradients(tokens, targets, weights, starts=starts, positions=positions)
    torch.cuda.synchronize()
    loss, wanted = by_autograd(model, tokens, targets, weights, starts, positions)
    # a mean over 1 000 positions of logits whose own error is 0.058 sqrt(3) of their size, about 0.3 (table 0.02, h of unit size over 256 elements)
    assert abs(float(model.loss.double().sum()) - loss) <= 0.01
    got = [model.grad_table, model.grad_proj] + ([model.grad_qkv] if heads else [])
    for x, want in zip(got, wanted):
        assert float((x.double() - want).norm() / want.norm()) <= 0.17
    assert int(model.status.item()) == 0


@pytest.mark.parametrize("logits", [True, False])
def test_a_step_in_a_replayed_graph_on_another_stream(logits):
    a, b = (TiedLm(300, 128, 700, heads=2, logits=logits) for _ in range(2))
    first = inputs(300, 700, 5)
    held = [t.clone() for t in (*first[0], *first[1])]
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        b.gradients(*held[:3], stream=s, starts=held[3], positions=held[4])
    for seed in range(3):
        batch_, (starts, positions) = inputs(300, 700, 10 + seed, 20 + 200 * seed)
        for h, t in zip(held, (*batch_, starts, positions)):
            h.copy_(t)
        a.gradients(*batch_, starts=starts, positions=positions)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("loss", "grad_table", "grad_proj", "grad_qkv"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_a_step_updates_every_parameter_and_reports_what_is_wrong():
    model = TiedLm(300, 128, 700, heads=4, logits=False)
    was = [t.clone() for t in (model.table, model.proj, model.qkv)]
    (tokens, targets, weights), (starts, positions) = inputs(300, 700, 6)
    model.step(tokens, targets, weights, starts=starts, positions=positions)
    for x, y in zip(was, (model.table, model.proj, model.qkv)):
        assert not torch.equal(x, y) and bool(torch.isfinite(y).all())
    assert int(model.status.item()) == 0
    starts[5], tokens[3], targets[9] = 701, 300, -3
    model.gradients(tokens, targets, weights, starts=starts, positions=positions)
    assert int(model.status.item()) == lmt.LMT_STATUS_BAD_SEQUENCE | lmt.LMT_STATUS_BAD_TOKEN | lmt.LMT_STATUS_BAD_TARGET
    with pytest.raises(ValueError):
        TiedLm(300, 100, 700, heads=3)
