"""Performance cases of the operators between the ends of a language model's training step, through the public Python calls.

    own                 whether run() makes the framework's calls or computes the plain form in elementary torch operations
    listed()            the cases that are tracked
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a training program holds before the call: tensors on the GPU, workspaces, results of the forward pass
    run(state)          one pass; returns everything the pass computed (whole buffers, no copies)
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs in 64 bits

The operators, for rows (tokens) with heads of D elements:

    rotary       every pair (a, b) of the first 2 F elements of a head becomes m (a cos - b sin, a sin + b cos) at the angle
                 position * frequency; pairs are neighbours, or lie F apart; the rest of the head is copied.  `inverse` turns
                 back: the gradient.
    attend       rows in sequences of unlike lengths, in one tensor with or without gaps.  s = scale q_i k_j, then
                 cap tanh(s / cap), then - slope |i - j|; i sees the j of its own sequence, with `causal` those up to itself,
                 with prefixes also all of its sequence's first ones.  out = softmax(s) v, lse = log sum exp(s).  Rows of no
                 sequence: out 0, lse -inf.  Consecutive query heads share a head of k and v.
    attend_grad  gradients of q, k and v from that of out; 0 for rows of no sequence
    linear_loss  logits = x table^T, never kept as a whole; per row lse, loss = w (lse - logit of the target), and the gradients of
                 x and table; rows whose target is the ignored one have none

A model is BERT-shaped: hidden sizes of 768 and 1024, heads of 64, 30 522 word pieces, sequences of up to 512 of unlike lengths;
longer sequences, wider heads, shared ones and other vocabularies are generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_IGNORE = -100
_CAP = 30.0


def _attend(name, op, **given):
    c = dict(op=op, layout="packed", sequences=1, longest=128, lengths="full", pick=0, spare=0, heads=12, kv_heads=12, size=64, dtype="bf16", causal=False, prefix=False, slopes=False, cap=0.0)
    return dict(c, **given) if name is None else dict(c, name=name, **given)


def listed():
    return [
        # queries and keys of one short sequence: the launch is all it costs
        dict(name="rotary_short", op="rotary", rows=37, heads=8, size=64, pairs=32, layout="half", dtype="bf16", far=512, magnitude=1.0, inverse=False),
        # queries and keys of 64 sequences of 512, 16 heads of each
        dict(name="rotary_large", op="rotary", rows=32768, heads=32, size=64, pairs=32, layout="half", dtype="bf16", far=512, magnitude=1.0, inverse=False),
        # the gradient behind it for half of wider heads, neighbours paired, positions stretched far beyond what was trained
        dict(name="rotary_back_far", op="rotary", rows=8192, heads=18, size=128, pairs=32, layout="neighbours", dtype="f16", far=1_000_000, magnitude=1.2, inverse=True),
        # one short sequence of a small model
        _attend("attend_short", "attend", longest=37, heads=4, kv_heads=4),
        # BERT-Base at 16 sequences of up to 512 a GPU, each in 512 rows
        _attend("attend_padded", "attend", layout="padded", sequences=16, longest=512, lengths="even", pick=1),
        # documents of a prefix and what follows from it, scores that fall with the distance, an odd head size
        _attend("attend_prefix", "attend", sequences=24, longest=1500, lengths="log", pick=2, spare=100, heads=10, kv_heads=5, size=72, dtype="f16", causal=True, prefix=True, slopes=True),
        # one long document, eight query heads to a key head, capped scores
        _attend("attend_long", "attend", longest=8192, heads=16, kv_heads=2, size=128, causal=True, cap=_CAP),
        # two short sequences of a small model in fp16
        _attend("attend_grad_short", "attend_grad", sequences=2, longest=50, lengths="even", pick=3, heads=4, kv_heads=4, dtype="f16"),
        # BERT-Large's heads, 32 768 tokens of sequences of up to 512 without padding
        _attend("attend_grad_packed", "attend_grad", sequences=128, longest=512, lengths="even", pick=4, heads=16, kv_heads=16),
        # one long document behind shared heads
        _attend("attend_grad_long", "attend_grad", longest=8192, heads=16, kv_heads=2, size=128, causal=True),
        # the masked positions of one sequence of a small model
        dict(name="linear_loss_small", op="linear_loss", rows=76, classes=2003, width=257, dtype="f16", ignored=0.1, weights=True, gradients=True),
        # every position of 16 sequences of 512 of BERT-Large, one in seven counted nowhere
        dict(name="linear_loss_large", op="linear_loss", rows=8192, classes=30522, width=1024, dtype="bf16", ignored=0.15, weights=True, gradients=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotary(rng, dtype):
    size = rng.choice((64, 64, 128, 2 * _log_int(rng, 4, 64)))
    pairs = rng.choice((size // 2, size // 2, size // 4, rng.randint(1, size // 2)))
    heads = rng.choice((1, 2, 4, 8, 12, 20, 24, 32, rng.randint(1, 32)))
    return dict(op="rotary", rows=_log_int(rng, 1, min(65536, 32768 * 32 * 64 // (heads * size))), heads=heads, size=size, pairs=max(1, pairs),
                layout=rng.choice(("half", "neighbours")), dtype=rng.choice((dtype, "f32")), far=_log_int(rng, 512, 4_000_000), magnitude=rng.choice((1.0, 1.0, 1.2)), inverse=rng.random() < 0.4)


def _draw_attend(rng, dtype, op):
    while True:     # gradients from 8 positions on: those of the queries and keys of a single one are nothing but rounding
        kv = rng.choice((1, 2, 4, 8, 12, 16, rng.randint(1, 16)))
        causal = rng.random() < 0.5
        c = _attend(None, op, layout=rng.choice(("packed", "packed", "padded")), sequences=rng.choice((1, 2, 16, 32, _log_int(rng, 1, 200))), longest=_log_int(rng, 1 if op == "attend" else 8, 8192),
                    lengths=rng.choice(("full", "even", "even", "log")), pick=rng.randrange(1_000_000), spare=rng.choice((0, 0, rng.randint(1, 200))),
                    heads=kv * rng.choice((1, 1, 1, 2, 4, 8)), kv_heads=kv, size=rng.choice((64, 64, 64, 128, 128, 32, rng.randint(8, 128))), dtype=dtype, causal=causal,
                    prefix=causal and rng.random() < 0.3, slopes=rng.random() < 0.3, cap=rng.choice((0.0, 0.0, 0.0, _CAP)))
        if c["heads"] > 32 or c["sequences"] * c["heads"] * c["longest"] ** 2 > 1_100_000_000 or c["sequences"] * c["longest"] * c["heads"] * c["size"] > 70_000_000:
            continue
        if work(c)["flops"] <= work(_attend(None, "attend_grad", longest=8192, heads=16, kv_heads=2, size=128, causal=True))["flops"]:
            return c


def draw(rng):
    op = rng.choice(("rotary", "attend", "attend", "attend_grad", "attend_grad", "linear_loss"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "rotary":
        return _draw_rotary(rng, dtype)
    if op != "linear_loss":
        return _draw_attend(rng, dtype, op)
    while True:
        width = rng.choice((128, 256, 512, 768, 1024, 1536, 2048, _log_int(rng, 33, 2050)))
        rows, classes = _log_int(rng, 4, 16384), rng.choice((30522, _log_int(rng, 50, 130000)))
        if rows * classes * width <= 8192 * 30522 * 1024 and rows * classes <= 300_000_000:
            return dict(op=op, rows=rows, classes=classes, width=width, dtype=dtype, ignored=rng.choice((0.0, 0.15, 0.85)), weights=rng.random() < 0.7, gradients=rng.random() < 0.75)


# ---- sequences ---------------------------------------------------------------


def _lengths(case):
    """The sequences' lengths: all the longest, evenly spread below it, or evenly over the logarithm.  The first one is the longest."""
    rng, n, top = random.Random(case["pick"]), case["sequences"], case["longest"]
    if case["lengths"] == "full":
        return [top] * n
    return [top] + [rng.randint(1, top) if case["lengths"] == "even" else _log_int(rng, 1, top) for _ in range(n - 1)]


def _starts(case):
    starts = [0]
    for length in _lengths(case):
        starts.append(starts[-1] + (case["longest"] if case["layout"] == "padded" else length))
    return starts


def _prefixes(case):
    rng = random.Random(case["pick"] + 1)
    return [rng.randint(0, length) for length in _lengths(case)]


def _rows(case):
    return _starts(case)[-1] + case["spare"]


def _pairs(case):
    """How many (i, j) are seen, a head."""
    total = 0
    for length, prefix in zip(_lengths(case), _prefixes(case) if case["prefix"] else [0] * case["sequences"]):
        total += length * length if not case["causal"] else length * (length + 1) // 2 + prefix * (prefix - 1) // 2
    return total


# ---- inputs ------------------------------------------------------------------


def _normal(g, shape, dtype, sigma):
    return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)


def _frequencies(case):
    """Of each pair of a rotary head, for a base of 10 000; slow pairs slowed further where positions go beyond what was trained."""
    f = 10000.0 ** (-torch.arange(case["pairs"], dtype=torch.float64) / case["pairs"])
    if case["far"] > 8192:
        turns = 8192 * f / (2 * math.pi)
        f = torch.where(turns > 8, f, f * 8192 / case["far"])
    return f.float().cuda()


def _whole(s, name, dtype):
    """A projection's output for q, k and v in one, and its three parts."""
    case = s["case"]
    H, G, D = case["heads"], case["kv_heads"], case["size"]
    s[name] = dtype if torch.is_tensor(dtype) else torch.empty((_rows(case), H + 2 * G, D), dtype=dtype, device="cuda")
    return s[name][:, :H], s[name][:, H:H + G], s[name][:, H + G:]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, dtype = case["op"], _DT[case["dtype"]]
    s = dict(case=case, workspace=None)
    if op == "rotary":
        s["x"] = _normal(g, (case["rows"], case["heads"], case["size"]), dtype, 1.0)
        s["positions"] = torch.randint(case["far"], (case["rows"],), generator=g, device="cuda")
        s["frequencies"], s["out"] = _frequencies(case), torch.empty_like(s["x"])
    elif op == "linear_loss":
        n, V, W = case["rows"], case["classes"], case["width"]
        s["x"], s["table"] = _normal(g, (n, W), dtype, 1.0), _normal(g, (V, W), dtype, 2.0 / math.sqrt(W))
        t = torch.randint(V, (n,), generator=g, device="cuda")
        s["targets"] = torch.where(torch.rand(n, generator=g, device="cuda") < case["ignored"], _IGNORE, t)
        s["weights"] = (0.5 + torch.rand(n, generator=g, device="cuda")) * (1.0 if case["dtype"] == "f16" else 1.0 / n) if case["weights"] else None
        s["loss"], s["lse"] = (torch.empty(n, device="cuda") for _ in range(2))
        s["grad_x"], s["grad_table"] = (torch.empty_like(s[x]) if case["gradients"] else None for x in ("x", "table"))
    else:
        T, H, G, D = _rows(case), case["heads"], case["kv_heads"], case["size"]
        s["q"], s["k"], s["v"] = _whole(s, "qkv", _normal(g, (T, H + 2 * G, D), dtype, 1.0))
        s["starts"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda")
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["layout"] == "padded" else None
        s["prefixes"] = torch.tensor(_prefixes(case), dtype=torch.int32, device="cuda") if case["prefix"] else None
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda") if case["slopes"] else None
        s["out"], s["lse"] = torch.empty((T, H, D), dtype=dtype, device="cuda"), torch.empty((H, T), device="cuda")
        if op == "attend_grad":
            out, lse = _plain_attend(s)
            s["out"].copy_(out), s["lse"].copy_(lse)
            s["grad_out"] = _normal(g, (T, H, D), dtype, 1e-2)
            s["grad_q"], s["grad_k"], s["grad_v"] = _whole(s, "grad_qkv", dtype)
    if own:  # what the framework's calls work in is kept by the program that makes them
        s["workspace"] = _workspace(case)
    return s


def _workspace(case):
    from paper_2402_02447_amd import lmt
    if case["op"] == "attend_grad":
        n = lmt.attention_grad_workspace(_rows(case), case["heads"], case["kv_heads"], case["size"])
    elif case["op"] == "linear_loss":
        n = lmt.linear_cross_entropy_workspace(case["rows"], case["classes"], case["width"], case["gradients"])
    else:
        return None
    return torch.empty(n, dtype=torch.uint8, device="cuda")


# ---- the plain forms ---------------------------------------------------------


def _plain_rotary(s):
    case, x = s["case"], s["x"].float()
    F = case["pairs"]
    angle = s["positions"].double().unsqueeze(1) * s["frequencies"].double()
    sin, cos = ((f(angle) * case["magnitude"]).float().unsqueeze(1) for f in (torch.sin, torch.cos))
    if case["inverse"]:
        sin = -sin
    if case["layout"] == "half":
        a, b = x[..., :F], x[..., F:2 * F]
        parts = (a * cos - b * sin, a * sin + b * cos, x[..., 2 * F:])
    else:
        a, b = x[..., :2 * F:2], x[..., 1:2 * F:2]
        parts = (torch.stack((a * cos - b * sin, a * sin + b * cos), 3).flatten(2), x[..., 2 * F:])
    return s["out"].copy_(torch.cat(parts, 2))


class _Padded:
    """Rows of sequences as [sequence][head][position] and back."""

    def __init__(self, s):
        case = s["case"]
        self.T, self.L, first = _rows(case), case["longest"], s["starts"][:-1].long()
        self.lengths = (s["starts"][1:] - s["starts"][:-1] if s["lengths"] is None else s["lengths"]).long()
        at = torch.arange(self.L, device="cuda")
        self.there = at < self.lengths.unsqueeze(1)
        self.rows = (first.unsqueeze(1) + at).clamp_(max=self.T - 1)
        row = torch.arange(self.T, device="cuda")
        self.of = torch.searchsorted(first, row, right=True) - 1
        self.pos = row - first[self.of]
        self.live = self.pos < self.lengths[self.of]
        self.pos = self.pos.clamp(max=self.L - 1)
        self.sees = self.there[:, None, None, :] & self.there[:, None, :, None]
        if case["causal"]:
            seen = at <= at.unsqueeze(1)
            if s["prefixes"] is not None:
                seen = seen | (at < s["prefixes"].long()[:, None, None, None])
            self.sees = self.sees & seen
        self.apart = (at - at.unsqueeze(1)).abs()

    def take(self, x, group=1):
        x = x.float()[self.rows].transpose(1, 2) * self.there[:, None, :, None]
        return x.repeat_interleave(group, 1) if group > 1 else x.contiguous()

    def back(self, x, rest=0.0):
        x = x.transpose(1, 2)[self.of, self.pos]
        return torch.where(self.live.view(-1, *([1] * (x.dim() - 1))), x, rest)


def _scores(s, P, q, k):
    """Scores, -inf where nothing is seen, and the derivative of the cap."""
    case = s["case"]
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(case["size"]))
    bend = None
    if case["cap"]:
        bend = torch.tanh_(x.div_(case["cap"]))
        x = bend * case["cap"]
    if s["slopes"] is not None:
        x = x - s["slopes"].view(-1, 1, 1) * P.apart
    return x.masked_fill_(~P.sees, -math.inf), bend


def _plain_attend(s):
    case, P = s["case"], _Padded(s)
    group = case["heads"] // case["kv_heads"]
    x, _ = _scores(s, P, P.take(s["q"]), P.take(s["k"], group))
    top = x.amax(3, keepdim=True).clamp_(min=-1e30)
    e = torch.exp_(x.sub_(top))
    total = e.sum(3, keepdim=True)
    out = torch.matmul(e, P.take(s["v"], group)) / total.clamp(min=1e-30)
    return P.back(out), P.back((top + torch.log(total)).squeeze(3), -math.inf).t()


def _plain_attend_grad(s):
    case, P = s["case"], _Padded(s)
    H, G, D = case["heads"], case["kv_heads"], case["size"]
    group = H // G
    q, k, v, go = P.take(s["q"]), P.take(s["k"], group), P.take(s["v"], group), P.take(s["grad_out"])
    x, bend = _scores(s, P, q, k)
    lse = torch.where(P.there.unsqueeze(1), s["lse"].t()[P.rows].transpose(1, 2), 0.0)
    p = torch.exp_(x.sub_(lse.unsqueeze(3)))
    delta = (go * P.take(s["out"])).sum(3, keepdim=True)
    grad_v = torch.matmul(p.transpose(2, 3).contiguous(), go)
    ds = torch.matmul(go, v.transpose(2, 3).contiguous()).sub_(delta).mul_(p).mul_(1.0 / math.sqrt(D))
    if bend is not None:
        ds.mul_(1 - bend.square_())
    grad_q, grad_k = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q)
    s["grad_q"].copy_(P.back(grad_q))
    s["grad_k"].copy_(P.back(grad_k.unflatten(1, (G, group)).sum(2)))
    s["grad_v"].copy_(P.back(grad_v.unflatten(1, (G, group)).sum(2)))


def _plain_loss(s):
    case, x, w, t = s["case"], s["x"].float(), s["table"].float(), s["targets"]
    logits = x @ w.t()
    counted = t != _IGNORE
    by = counted.float() if s["weights"] is None else torch.where(counted, s["weights"], 0.0)
    top = logits.amax(1, keepdim=True)
    at = torch.where(counted, t, 0).unsqueeze(1)
    hit = logits.gather(1, at).squeeze(1)
    e = torch.exp_(logits.sub_(top))
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    out = {"loss": s["loss"].copy_(by * (lse - hit)), "lse": s["lse"].copy_(lse)}
    if case["gradients"]:
        d = e.mul_(by.unsqueeze(1) / total).scatter_add_(1, at, -by.unsqueeze(1))
        out |= {"grad_x": s["grad_x"].copy_(d @ w), "grad_table": s["grad_table"].copy_(d.t() @ x)}
    return out


def _plain(s):
    op = s["case"]["op"]
    if op == "rotary":
        return _plain_rotary(s)
    if op == "linear_loss":
        return _plain_loss(s)
    if op == "attend":
        out, lse = _plain_attend(s)
        return {"out": s["out"].copy_(out), "lse": s["lse"].copy_(lse)}
    _plain_attend_grad(s)
    return {x: s[x] for x in ("grad_q", "grad_k", "grad_v")}


def run(s):
    if not own:
        return _plain(s)
    from paper_2402_02447_amd import lmt
    case = s["case"]
    op = case["op"]
    if op == "rotary":
        lmt.rotary(s["x"], s["positions"], s["frequencies"], s["out"], neighbours=case["layout"] == "neighbours", magnitude=case["magnitude"], inverse=case["inverse"])
        return s["out"]
    if op == "linear_loss":
        lmt.linear_cross_entropy(s["x"], s["table"], s["targets"], s["workspace"], s["loss"], s["lse"], s["grad_x"], s["grad_table"], weights=s["weights"], ignore=_IGNORE)
        return {x: s[x] for x in ("loss", "lse", "grad_x", "grad_table") if s[x] is not None}
    masks = dict(lengths=s["lengths"], prefixes=s["prefixes"], slopes=s["slopes"], scale=1.0 / math.sqrt(case["size"]), cap=case["cap"], causal=case["causal"])
    if op == "attend":
        lmt.attention(s["q"], s["k"], s["v"], s["out"], s["lse"], s["starts"], **masks)
        return {"out": s["out"], "lse": s["lse"]}
    lmt.attention_grad(s["grad_out"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["grad_q"], s["grad_k"], s["grad_v"], s["workspace"], s["starts"], **masks)
    return {x: s[x] for x in ("grad_q", "grad_k", "grad_v")}


# ---- what a pass cannot do without -------------------------------------------


def work(case):
    op, size = case["op"], _SIZE[case["dtype"]]
    if op == "rotary":
        n = case["rows"] * case["heads"] * case["size"]
        return {"bytes": 2 * n * size + 8 * case["rows"] + 4 * case["pairs"], "flops": 6 * case["rows"] * case["heads"] * case["pairs"]}
    if op == "linear_loss":
        n, V, W = case["rows"], case["classes"], case["width"]
        sides = 2 if case["gradients"] else 1
        return {"bytes": sides * (n + V) * W * size + n * 20, "flops": (6 if case["gradients"] else 2) * n * V * W}
    T, H, G, D = sum(_lengths(case)), case["heads"], case["kv_heads"], case["size"]
    rows = _rows(case)
    if op == "attend":
        return {"bytes": T * (H + 2 * G) * D * size + rows * H * (D * size + 4), "flops": 4 * D * H * _pairs(case)}
    return {"bytes": T * (3 * H + 2 * G) * D * size + T * H * 4 + rows * (H + 2 * G) * D * size, "flops": 10 * D * H * _pairs(case)}


# ---- 64 bits -----------------------------------------------------------------


def _exact_rotary(case, s):
    F, x = case["pairs"], s["x"].double()
    turn = torch.polar(torch.full((case["rows"], F), case["magnitude"], dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["frequencies"].double()[None])
    turn = (turn.conj() if case["inverse"] else turn).unsqueeze(1)
    out, lo, hi = x.clone(), slice(0, F), slice(F, 2 * F)
    if case["layout"] != "half":
        lo, hi = slice(0, 2 * F, 2), slice(1, 2 * F, 2)
    z = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * turn
    out[..., lo], out[..., hi] = z.real, z.imag
    return out


def _exact_attend(case, s, want_grad):
    """Sequence by sequence and head by head, from the definition."""
    T, H, G, D = _rows(case), case["heads"], case["kv_heads"], case["size"]
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros((T, H, D), **f64), torch.full((H, T), -math.inf, **f64)
    grads = [torch.zeros((T, n, D), **f64) for n in (H, G, G)]
    prefixes = _prefixes(case) if case["prefix"] else [0] * case["sequences"]
    for first, n, prefix in zip(_starts(case), _lengths(case), prefixes):
        if n == 0:
            continue
        i = torch.arange(n, device="cuda")
        hidden = (i[None, :] > i[:, None]) & (i[None, :] >= prefix) if case["causal"] else None
        away = (i[None, :] - i[:, None]).abs().double()
        rows = slice(first, first + n)
        for h in range(H):
            q, k, v = (x[rows, n_h].double() for x, n_h in ((s["q"], h), (s["k"], h * G // H), (s["v"], h * G // H)))
            raw = torch.mm(q, k.t().contiguous()) / math.sqrt(D)
            x = case["cap"] * torch.tanh(raw / case["cap"]) if case["cap"] else raw
            if case["slopes"]:
                x = x - float(s["slopes"][h]) * away
            if hidden is not None:
                x = x.masked_fill(hidden, -math.inf)
            total = torch.logsumexp(x, 1)
            p = torch.exp(x - total[:, None])
            o = torch.mm(p, v)
            out[rows, h], lse[h, rows] = o, total
            if want_grad:
                go = s["grad_out"][rows, h].double()
                d = p * (torch.mm(go, v.t().contiguous()) - (go * o).sum(1, keepdim=True))
                if case["cap"]:
                    d = d / torch.cosh(raw / case["cap"]) ** 2
                d = d / math.sqrt(D)
                grads[0][rows, h] = torch.mm(d, k)
                grads[1][rows, h * G // H] += torch.mm(d.t().contiguous(), q)
                grads[2][rows, h * G // H] += torch.mm(p.t().contiguous(), go)
    return dict(zip(("grad_q", "grad_k", "grad_v"), grads)) if want_grad else {"out": out, "lse": lse}


def _exact_loss(case, s):
    n, V, W = case["rows"], case["classes"], case["width"]
    w, loss, lse = s["table"].double(), [], []
    grad_x, grad_w = (torch.zeros(shape, dtype=torch.float64, device="cuda") for shape in ((n, W), (V, W)))
    for lo in range(0, n, 1024):
        x, t = s["x"][lo:lo + 1024].double(), s["targets"][lo:lo + 1024]
        by = (t != _IGNORE).double() * (1.0 if s["weights"] is None else s["weights"][lo:lo + 1024].double())
        logits = torch.mm(x, w.t().contiguous())
        total = torch.logsumexp(logits, 1)
        hot = (torch.arange(V, device="cuda")[None, :] == t[:, None]).double()
        lse.append(total)
        loss.append(by * (total - (hot * logits).sum(1)))
        d = by[:, None] * (torch.exp(logits - total[:, None]) - hot)
        grad_x[lo:lo + 1024] = torch.mm(d, w)
        grad_w += torch.mm(d.t().contiguous(), x)
    out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    return out | {"grad_x": grad_x, "grad_table": grad_w} if case["gradients"] else out


def exact(case, seed):
    if case["op"].startswith("attend") and case["sequences"] * case["heads"] > 4000:
        return None     # a loop over so many sequences and heads takes too long
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    if case["op"] == "linear_loss":
        return _exact_loss(case, s)
    return _exact_attend(case, s, case["op"] == "attend_grad")
