"""Performance cases of the operators at the two ends of a language model's training step, through the public Python calls.

    own                 whether run() makes the framework's calls or computes the plain form in elementary torch operations
    listed()            the cases that are tracked
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a training program holds before the call: tensors on the GPU, workspaces, quantised operands
    run(state)          one pass; returns everything the pass computed (whole buffers, no copies)
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs in 64 bits

The operators, with T tokens, a vocabulary of V entries and rows of H elements:

    embed        out[t] = scale * table[token[t]]
    embed_grad   grad[v] = (the old grad[v], if it accumulates) + scale * sum over t with token[t] = v of grad_out[t]; no
                 gradient for the padding token
    quantize     8-bit floating point with a power of two for every 128 elements along a row ("row"), or for every square of 128 x 128
                 ("tile"): the smallest one that brings the block's largest magnitude to the type's largest value or below.
                 The matrix, its transpose (blocks along the columns), or both.  Rows are padded with zeros to whole blocks.
    product      c[m][n] = (the old c, if it accumulates) + sum over k of a[m][k] b[n][k], both operands as quantize gives them
    loss         per row i with target t and weight w: loss = w (lse(x) - x[t]), grad = w (softmax(x) - onehot(t)); rows
                 whose target is the ignored one have neither

A model is BERT-shaped: hidden sizes of 768 and 1024, feed-forward parts of 4x, 30 522 word pieces, sequences of up to 512,
16 sequences a GPU; small models and longer vocabularies are generic.  Word pieces follow Zipf's law over a shuffled vocabulary;
`mask` and `pad` of the tokens are the mask's and the padding's, as masked language modelling makes them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2, "i32": 4, "i64": 8}
_F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_TOP = {"e4m3": (8, 3, -6), "e5m2": (15, 2, -14)}   # exponent of the largest value (1.75 * 2^it), mantissa bits, least normal exponent
_MASK_ID, _PAD_ID, _IGNORE = 103, 0, -100


def listed():
    return [
        # one short sequence looked up for a small model: the launch is all it costs
        dict(name="embed_short", op="embed", tokens=37, vocab=2000, width=256, dtype="f32", out="f32", ids="i64", scale=16.0, mask=0.15, pad=0.0),
        # the input of a large step: 64 sequences of 512, weights kept in fp32, activations in bf16
        dict(name="embed_large", op="embed", tokens=32768, vocab=30522, width=1024, dtype="f32", out="bf16", ids="i32", scale=32.0, mask=0.12, pad=0.25),
        # the gradient of a small model's table, a few short sequences, odd sizes
        dict(name="embed_grad_small", op="embed_grad", tokens=611, vocab=2003, width=257, dtype="f32", grad="f32", ids="i64", scale=16.0, mask=0.15, pad=0.1, accumulate=False),
        # BERT-Base at 16 sequences of 512 a GPU: the dense gradient that a clipped bucket reads
        dict(name="embed_grad_base", op="embed_grad", tokens=8192, vocab=30522, width=768, dtype="bf16", grad="f32", ids="i64", scale=1.0, mask=0.12, pad=0.25, accumulate=False),
        # tied weights: added to what the output layer has left there; half a thousand sequences, long runs of one token
        dict(name="embed_grad_tied", op="embed_grad", tokens=262144, vocab=30522, width=1024, dtype="bf16", grad="f32", ids="i32", scale=1.0, mask=0.12, pad=0.25, accumulate=True),
        # activations for the forward product and for the weight gradient behind it, read once
        dict(name="quantize_activation", op="quantize", rows=8192, cols=1024, dtype="bf16", fp8="e4m3", blocks="row", sides="both"),
        # the tied weights after an optimizer step, for the logits and for the gradient of their input
        dict(name="quantize_weights", op="quantize", rows=30522, cols=1024, dtype="f32", fp8="e4m3", blocks="tile", sides="both"),
        # a projection of one short sequence
        dict(name="product_short", op="product", m=37, n=1024, k=1024, a="e4m3", b="e4m3", c="bf16", accumulate=False),
        # logits of the masked positions of 32 sequences (76 each): an odd number of columns
        dict(name="product_logits", op="product", m=2432, n=30522, k=1024, a="e4m3", b="e4m3", c="bf16", accumulate=False),
        # gradient of a feed-forward matrix over 32 768 tokens: few tiles and a long sum, added to the bucket's fp32 gradient
        dict(name="product_weight_grad", op="product", m=4096, n=1024, k=32768, a="e5m2", b="e4m3", c="f32", accumulate=True),
        # the loss of a few masked positions in fp32
        dict(name="loss_few", op="loss", rows=19, classes=30522, dtype="f32", ids="i64", ignored=0.1, weights=True),
        # every position of 32 sequences of 512 with its gradient, one in seven of them counted nowhere
        dict(name="loss_large", op="loss", rows=16384, classes=30522, dtype="bf16", ids="i64", ignored=0.15, weights=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return rng.choice((rng.choice((128, 256, 384, 512, 768, 1024, 1536, 2048)), _log_int(rng, 33, 2050)))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "embed_grad", "quantize", "product", "product", "loss"))
    dtype, ids = rng.choice(("f32", "f16", "bf16", "bf16")), rng.choice(("i32", "i64"))
    mask, pad = rng.choice((0.0, 0.12, 0.15)), rng.choice((0.0, 0.1, 0.25, 0.5))
    if op == "embed" or op == "embed_grad":
        width, vocab = _width(rng), _log_int(rng, 300, 60000)
        tokens = _log_int(rng, 1, min(262144, (32768 if op == "embed" else 262144) * 1024 // width))
        c = dict(op=op, tokens=tokens, vocab=vocab, width=width, dtype=dtype, ids=ids, scale=rng.choice((1.0, 0.5, round(math.sqrt(width), 3))), mask=mask, pad=pad)
        return dict(c, out=rng.choice(("bf16", "f16", "f32"))) if op == "embed" else dict(c, grad=rng.choice(("f32", "f32", "bf16", "f16")), accumulate=rng.random() < 0.4)
    if op == "quantize":
        cols = rng.choice((_width(rng), 4 * _width(rng)))
        return dict(op=op, rows=_log_int(rng, 1, min(65536, 30_000_000 // cols)), cols=cols, dtype=dtype, fp8=rng.choice(("e4m3", "e4m3", "e5m2")),
                    blocks=rng.choice(("row", "row", "tile")), sides=rng.choice(("both", "rows", "cols")))
    if op == "product":
        while True:
            m, n, k = _log_int(rng, 1, 32768), _log_int(rng, 64, 32768), _log_int(rng, 64, 32768)
            if m * n * k <= 4096 * 1024 * 32768 and m * n <= 100_000_000 and (m + n) * k <= 200_000_000:
                break
        a, b = rng.choice((("e4m3", "e4m3"), ("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e5m2", "e5m2")))
        return dict(op=op, m=m, n=n, k=k, a=a, b=b, c=rng.choice(("bf16", "bf16", "f32", "f16")), accumulate=rng.random() < 0.3)
    classes = _log_int(rng, 2, 130000)
    return dict(op=op, rows=_log_int(rng, 1, min(32768, 16384 * 30522 // classes // (2 if dtype == "f32" else 1))), classes=classes, dtype=dtype, ids=ids,
                ignored=rng.choice((0.0, 0.15, 0.85)), weights=rng.random() < 0.7)


# ---- inputs ------------------------------------------------------------------


def _tokens(g, case):
    """Zipf over a shuffled vocabulary; then the mask's and the padding's tokens."""
    n, V = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    ids = torch.randperm(V, generator=g, device="cuda")[rank]
    kind = torch.rand(n, generator=g, device="cuda")
    ids = torch.where(kind < case["mask"], min(_MASK_ID, V - 1), ids)
    ids = torch.where(kind >= 1 - case["pad"], _PAD_ID, ids)
    return ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _normal(g, shape, dtype, sigma):
    return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)


def _blocks(cols):
    return -(-cols // 128)


def _scale_bytes(cols):
    return -(-cols // 512) * 4


def _operand(g, rows, cols, fp8):
    """A quantised matrix as quantize leaves it: activations or weights of rows of unlike sizes (e4m3), or gradients (e5m2)."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    x *= torch.exp(torch.randn((rows, 1), generator=g, device="cuda")) * (1e-3 if fp8 == "e5m2" else 0.1)
    q, s = _quantised(x, fp8, "row")
    return q, s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    s = dict(case=case)
    if op == "embed":
        s["table"] = _normal(g, (case["vocab"], case["width"]), _DT[case["dtype"]], 0.02)
        s["tokens"] = _tokens(g, case)
        s["out"] = torch.empty((case["tokens"], case["width"]), dtype=_DT[case["out"]], device="cuda")
    elif op == "embed_grad":
        s["grad_out"] = _normal(g, (case["tokens"], case["width"]), _DT[case["dtype"]], 1e-2 if case["dtype"] == "f16" else 1e-3)
        s["tokens"] = _tokens(g, case)
        s["grad"] = _normal(g, (case["vocab"], case["width"]), _DT[case["grad"]], 1e-3)
    elif op == "quantize":
        r, c, dt = case["rows"], case["cols"], _F8[case["fp8"]]
        x = torch.randn((r, c), generator=g, device="cuda") * torch.exp(0.5 * torch.randn((1, c), generator=g, device="cuda"))
        s["x"] = x.to(_DT[case["dtype"]])
        if case["sides"] != "cols":
            s["q"] = torch.empty((r, 128 * _blocks(c)), dtype=dt, device="cuda")
            s["scales"] = torch.empty((r, _scale_bytes(c)), dtype=torch.uint8, device="cuda")
        if case["sides"] != "rows":
            s["qt"] = torch.empty((c, 128 * _blocks(r)), dtype=dt, device="cuda")
            s["scales_t"] = torch.empty((c, _scale_bytes(r)), dtype=torch.uint8, device="cuda")
    elif op == "product":
        s["a"], s["a_scales"] = _operand(g, case["m"], case["k"], case["a"])
        s["b"], s["b_scales"] = _operand(g, case["n"], case["k"], case["b"])
        size = 1e-4 if "e5m2" in (case["a"], case["b"]) else 1e-2
        s["c"] = _normal(g, (case["m"], case["n"]), _DT[case["c"]], size) if case["accumulate"] else torch.empty((case["m"], case["n"]), dtype=_DT[case["c"]], device="cuda")
    else:
        n, V = case["rows"], case["classes"]
        s["logits"] = _normal(g, (n, V), _DT[case["dtype"]], 2.0)
        t = torch.randint(V, (n,), generator=g, device="cuda")
        t = torch.where(torch.rand(n, generator=g, device="cuda") < case["ignored"], _IGNORE, t)
        s["targets"] = t.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        s["weights"] = (0.5 + torch.rand(n, generator=g, device="cuda")) / n if case["weights"] else None
        s["loss"], s["lse"] = (torch.empty(n, device="cuda") for _ in range(2))
        s["grad"] = torch.empty_like(s["logits"])
    # what the framework's calls work in is kept by the program that makes them
    s["workspace"] = torch.empty(_workspace_bytes(case), dtype=torch.uint8, device="cuda") if own and op in ("embed_grad", "product") else None
    return s


def _workspace_bytes(case):
    from paper_2402_02447_amd import lmt
    if case["op"] == "embed_grad":
        return lmt.embed_grad_workspace(case["tokens"], case["vocab"], case["width"])
    return lmt.matmul_workspace(case["m"], case["n"], case["k"])


# ---- the plain forms ---------------------------------------------------------


def _quantised(x, fp8, blocks):
    """x (fp32) in 8 bits and its scales' exponents, biased by 127, rows padded to whole blocks."""
    rows, cols = x.shape
    nb = _blocks(cols)
    y = torch.nn.functional.pad(x, (0, 128 * nb - cols))
    size = y.abs().reshape(rows, nb, 128).amax(2)
    if blocks == "tile":
        rb = _blocks(rows)
        size = torch.nn.functional.pad(size, (0, 0, 0, 128 * rb - rows)).reshape(rb, 128, nb).amax(1)
        size = size.repeat_interleave(128, 0)[:rows]
    part, power = torch.frexp(size)                      # size = part * 2^power, 1/2 <= part < 1
    e = power - 1 - _TOP[fp8][0] + (part > 0.875)
    e = torch.where(size == 0, -126, e).clamp_(min=-126)
    q = torch.ldexp(y.reshape(rows, nb, 128), -e.unsqueeze(2)).reshape(rows, 128 * nb).to(_F8[fp8])
    scales = torch.full((rows, _scale_bytes(cols)), 127, dtype=torch.uint8, device=x.device)
    scales[:, :nb] = (e + 127).to(torch.uint8)
    return q, scales


def _values(q, scales):
    rows, cols = q.shape
    e = scales[:, : cols // 128].to(torch.int32) - 127
    return torch.ldexp(q.float().reshape(rows, cols // 128, 128), e.unsqueeze(2)).reshape(rows, cols)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "embed":
        return (s["table"][s["tokens"]].float() * case["scale"]).to(s["out"].dtype)
    if op == "embed_grad":
        t = s["tokens"]
        rows = s["grad_out"].float() * ((t != _PAD_ID).float() * case["scale"]).unsqueeze(1)
        total = s["grad"].float() if case["accumulate"] else torch.zeros(s["grad"].shape, device="cuda")
        if total.data_ptr() == s["grad"].data_ptr():
            return total.index_add_(0, t, rows)
        return s["grad"].copy_(total.index_add_(0, t, rows))
    if op == "quantize":
        x, out = s["x"].float(), {}
        if case["sides"] != "cols":
            out["q"], out["scales"] = _quantised(x, case["fp8"], case["blocks"])
        if case["sides"] != "rows":
            out["qt"], out["scales_t"] = _quantised(x.t().contiguous(), case["fp8"], case["blocks"])
        return out
    if op == "product":
        c = _values(s["a"], s["a_scales"]) @ _values(s["b"], s["b_scales"]).t()
        return s["c"].copy_(c + s["c"].float() if case["accumulate"] else c)
    x, t = s["logits"].float(), s["targets"].long()
    counted = t != _IGNORE
    w = counted.float() if s["weights"] is None else torch.where(counted, s["weights"], 0.0)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    at = torch.where(counted, t, 0).unsqueeze(1)
    loss = w * (lse - x.gather(1, at).squeeze(1))
    grad = (e / total * w.unsqueeze(1)).scatter_add_(1, at, -w.unsqueeze(1))
    return {"loss": loss, "lse": lse, "grad": grad.to(s["logits"].dtype)}


def run(s):
    if not own:
        return _plain(s)
    from paper_2402_02447_amd import lmt
    case = s["case"]
    op = case["op"]
    if op == "embed":
        lmt.embed(s["table"], s["tokens"], s["out"], scale=case["scale"])
        return s["out"]
    if op == "embed_grad":
        lmt.embed_grad(s["grad_out"], s["tokens"], s["grad"], s["workspace"], scale=case["scale"], skip_token=_PAD_ID, accumulate=case["accumulate"])
        return s["grad"]
    if op == "quantize":
        lmt.quantize(s["x"], s.get("q"), s.get("scales"), s.get("qt"), s.get("scales_t"), tile=case["blocks"] == "tile")
        return {k: s[k] for k in ("q", "scales", "qt", "scales_t") if k in s}
    if op == "product":
        lmt.matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], s["c"], s["workspace"], accumulate=case["accumulate"])
        return s["c"]
    lmt.cross_entropy(s["logits"], s["targets"], s["loss"], s["lse"], s["grad"], weights=s["weights"], ignore=_IGNORE)
    return {k: s[k] for k in ("loss", "lse", "grad")}


# ---- what a pass cannot do without -------------------------------------------


def _distinct(case, n):
    """How many different entries n Zipf draws from the vocabulary touch on average, the mask's and the padding's beside them."""
    V = case["vocab"]
    edge = torch.log(torch.arange(1, V + 2, dtype=torch.float64)) / math.log(V + 1)
    p = edge[1:] - edge[:-1]
    return min(n, float((1 - torch.exp(n * (1 - case["mask"] - case["pad"]) * torch.log1p(-p))).sum()) + 1)


def work(case):
    op = case["op"]
    if op == "embed":
        T, H = case["tokens"], case["width"]
        return {"bytes": T * _SIZE[case["ids"]] + _distinct(case, T) * H * _SIZE[case["dtype"]] + T * H * _SIZE[case["out"]], "flops": T * H}
    if op == "embed_grad":
        T, H, V, kept = case["tokens"], case["width"], case["vocab"], 1 - case["pad"]
        table = 2 * _distinct(case, T) if case["accumulate"] else V
        return {"bytes": T * _SIZE[case["ids"]] + kept * T * H * _SIZE[case["dtype"]] + table * H * _SIZE[case["grad"]], "flops": kept * T * H}
    if op == "quantize":
        n, sides = case["rows"] * case["cols"], 2 if case["sides"] == "both" else 1
        return {"bytes": n * _SIZE[case["dtype"]] + sides * n * (1 + 1 / 128), "flops": n * (1 + sides)}
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * k * (1 + 1 / 128) + m * n * _SIZE[case["c"]] * (2 if case["accumulate"] else 1), "flops": 2 * m * n * k}
    n, kept = case["rows"] * case["classes"], 1 - case["ignored"]
    return {"bytes": 2 * n * _SIZE[case["dtype"]] + case["rows"] * (12 + _SIZE[case["ids"]]), "flops": 5 * kept * n}


# ---- 64 bits -----------------------------------------------------------------


def _fp8_nearest(y, fp8):
    """y rounded to the type's nearest value, ties to even, in 64 bits."""
    _, bits, least = _TOP[fp8]
    e = torch.floor(torch.log2(y.abs().clamp(min=1e-300))).clamp_(min=least)
    unit = torch.exp2(e - bits)
    return torch.round(y / unit) * unit


def _exact_quantised(x, fp8, tile):
    rows, cols = x.shape
    most = 1.75 * 2.0 ** _TOP[fp8][0]
    nr, nc = -(-rows // 128), -(-cols // 128)
    z = torch.zeros((128 * nr, 128 * nc), dtype=torch.float64, device=x.device)
    z[:rows, :cols] = x
    if tile:
        size = z.abs().view(nr, 128, nc, 128).amax((1, 3)).repeat_interleave(128, 0)
    else:
        size = z.abs().view(128 * nr, nc, 128).amax(2)
    e = torch.ceil(torch.log2((size / most).clamp(min=2.0 ** -126)))
    z /= torch.exp2(e).repeat_interleave(128, 1)
    return _fp8_nearest(z, fp8)[:rows].float()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        return torch.index_select(s["table"].double(), 0, s["tokens"].long()) * case["scale"]
    if op == "embed_grad":
        t = s["tokens"].long()
        order = torch.argsort(t, stable=True)
        order = order[t[order] != _PAD_ID]
        key = t[order]
        total = s["grad"].double() if case["accumulate"] else torch.zeros(s["grad"].shape, dtype=torch.float64, device="cuda")
        width = max(1, 100_000_000 // max(1, case["tokens"]))
        for lo in range(0, case["width"], width):           # running sums along the sorted tokens, differences at the ends of runs
            run_sum = torch.cumsum(s["grad_out"][:, lo:lo + width].double()[order], 0)
            if key.numel():
                end = torch.nonzero(torch.cat([key[1:] != key[:-1], torch.ones(1, dtype=torch.bool, device="cuda")])).squeeze(1)
                part = run_sum[end]
                part[1:] -= run_sum[end[:-1]]
                total[key[end], lo:lo + width] += part * case["scale"]
        return total
    if op == "quantize":
        x, out = s["x"].double(), {}
        if case["sides"] != "cols":
            out |= {"q": _exact_quantised(x, case["fp8"], case["blocks"] == "tile"), "scales": None}
        if case["sides"] != "rows":
            out |= {"qt": _exact_quantised(x.t(), case["fp8"], case["blocks"] == "tile"), "scales_t": None}
        return out
    if op == "product":
        def wide(q, scales):
            return q.double() * torch.exp2(scales[:, : q.shape[1] // 128].double() - 127).repeat_interleave(128, 1)
        c = torch.mm(wide(s["a"], s["a_scales"]), wide(s["b"], s["b_scales"]).t().contiguous())
        return c + s["c"].double() if case["accumulate"] else c
    loss, lse, grad = [], [], torch.empty(s["logits"].shape, dtype=torch.float64 if s["logits"].numel() <= 200_000_000 else torch.float32, device="cuda")
    for lo in range(0, case["rows"], 1024):
        x, t = s["logits"][lo:lo + 1024].double(), s["targets"][lo:lo + 1024].long()
        w = torch.ones(x.shape[0], dtype=torch.float64, device="cuda") if s["weights"] is None else s["weights"][lo:lo + 1024].double()
        w = w * (t != _IGNORE)
        l = torch.logsumexp(x, 1)
        hot = torch.arange(case["classes"], device="cuda").unsqueeze(0) == t.unsqueeze(1)
        lse.append(l)
        loss.append(w * (l - torch.where(hot, x, 0.0).sum(1)))
        grad[lo:lo + 1024] = (w.unsqueeze(1) * (torch.exp(x - l.unsqueeze(1)) - hot.double())).to(grad.dtype)
    return {"loss": torch.cat(loss), "lse": torch.cat(lse), "grad": grad}
