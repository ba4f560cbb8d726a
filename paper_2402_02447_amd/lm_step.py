"""A small language model trained with the library's calls from end to end: the operators of lmt.h around the clip and Adam.

The model predicts each token's successor: x = scale * table[tokens], h = x P^T, logits = h table^T, with the table tied (input
and output).  One step is
    embed, quantize, matmul                        forward, operands in 8 bits
    cross_entropy                                  mean loss of the counted positions; the gradient in the logits' place
    quantize, matmul                               gradients of h, x, P and, through the output, of the table
    embed_grad                                     added to the table's gradient: tokens sorted, no gradient for the padding
    bucket_clip_adam                               the parameters' update, bucket by bucket
with nothing but these calls on the stream: every buffer is allocated beforehand.

Run as ``python -m paper_2402_02447_amd.lm_step`` (needs a GPU): prints the loss of some steps on a made-up language."""
from __future__ import annotations

import argparse
import math
from typing import List

import torch

from . import lmt
from .binding import BCA_GRAD_F32, AdamHyper, Plan, alg1_thresholds
from .buckets import whole_tensors

PADDING = 0
IGNORE = -100


class _Fp8:
    """A matrix in 8 bits and its transpose, with the scales of both."""

    def __init__(self, rows: int, cols: int, dtype, tile: bool = False):
        def pair(r, c):
            q, s = lmt.fp8_shapes(r, c)
            return torch.empty(q, dtype=dtype, device="cuda"), torch.empty(s, dtype=torch.uint8, device="cuda")
        (self.q, self.scales), (self.qt, self.scales_t), self.tile = pair(rows, cols), pair(cols, rows), tile

    def take(self, x, stream) -> None:
        lmt.quantize(x, self.q, self.scales, self.qt, self.scales_t, tile=self.tile, stream=stream)

    @property
    def rows(self):
        return self.q, self.scales

    @property
    def cols(self):
        return self.qt, self.scales_t


class TiedLm:
    """The model, its gradients, moments and everything a step works in, for `tokens` positions a step."""

    def __init__(self, vocab: int, width: int, tokens: int, seed: int = 0, clip: float = 1.0, hyper: AdamHyper = AdamHyper(lr=3e-3)):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.scale, self.hyper, self.step_count = math.sqrt(width), hyper, 0
        self.table = torch.randn(vocab, width, generator=g, device="cuda") * 0.02
        self.proj = torch.randn(width, width, generator=g, device="cuda") / math.sqrt(width)
        self.grad_table, self.grad_proj = torch.empty_like(self.table), torch.empty_like(self.proj)

        def bf16(rows, cols):
            return torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
        e4m3, e5m2 = torch.float8_e4m3fn, torch.float8_e5m2
        self.x, self.h, self.dh, self.dx, self.logits = (bf16(tokens, n) for n in (width, width, width, width, vocab))
        self.x8, self.h8 = _Fp8(tokens, width, e4m3), _Fp8(tokens, width, e4m3)
        self.table8, self.proj8 = _Fp8(vocab, width, e4m3, tile=True), _Fp8(width, width, e4m3, tile=True)
        self.dlogits8, self.dh8 = _Fp8(tokens, vocab, e5m2), _Fp8(tokens, width, e5m2)
        self.loss = torch.empty(tokens, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        need = [lmt.embed_grad_workspace(tokens, vocab, width)]
        need += [lmt.matmul_workspace(*mnk) for mnk in ((tokens, width, width), (tokens, vocab, width), (tokens, width, vocab), (vocab, width, tokens), (width, width, tokens))]
        self.workspace = torch.empty(max(need), dtype=torch.uint8, device="cuda")   # one call after the other on one stream: they share it

        tensors: List[torch.Tensor] = [self.table, self.proj]
        layout = whole_tensors([t.numel() for t in tensors], 1)                     # a bucket per tensor, the last one first
        self.moments = [[torch.zeros_like(t).view(-1) for t in tensors] for _ in range(2)]
        self.plan = Plan.from_layout(layout, BCA_GRAD_F32, device=torch.cuda.current_device())
        self.plan.bind([self.grad_table.view(-1), self.grad_proj.view(-1)], [t.view(-1) for t in tensors], *self.moments)
        self.thresholds = torch.from_numpy(alg1_thresholds(clip, layout.n_buckets)).cuda()

    def gradients(self, tokens, targets, weights, stream=None) -> None:
        """Loss (per position, weighted) and gradients of a batch.  tokens, targets: [tokens] int32 or int64; weights: [tokens]."""
        T, s = self, stream
        T.table8.take(T.table, s), T.proj8.take(T.proj, s)                          # weights as the last update left them
        lmt.embed(T.table, tokens, T.x, T.scale, T.status, s)
        T.x8.take(T.x, s)
        lmt.matmul(*T.x8.rows, *T.proj8.rows, T.h, T.workspace, stream=s)           # h = x P^T
        T.h8.take(T.h, s)
        lmt.matmul(*T.h8.rows, *T.table8.rows, T.logits, T.workspace, stream=s)     # logits = h table^T
        lmt.cross_entropy(T.logits, targets, T.loss, None, T.logits, weights, IGNORE, T.status, s)
        T.dlogits8.take(T.logits, s)
        lmt.matmul(*T.dlogits8.rows, *T.table8.cols, T.dh, T.workspace, stream=s)   # dh = dlogits table
        lmt.matmul(*T.dlogits8.cols, *T.h8.cols, T.grad_table, T.workspace, stream=s)   # dtable = dlogits^T h
        T.dh8.take(T.dh, s)
        lmt.matmul(*T.dh8.rows, *T.proj8.cols, T.dx, T.workspace, stream=s)         # dx = dh P
        lmt.matmul(*T.dh8.cols, *T.x8.cols, T.grad_proj, T.workspace, stream=s)     # dP = dh^T x
        lmt.embed_grad(T.dx, tokens, T.grad_table, T.workspace, T.scale, PADDING, True, T.status, s)

    def step(self, tokens, targets, weights, stream=None) -> None:
        self.gradients(tokens, targets, weights, stream)
        self.step_count += 1
        self.plan.bucket_clip_adam(self.thresholds, self.hyper, self.step_count, stream=stream)


def batch(vocab: int, tokens: int, generator):
    """Positions of a made-up language in which token t is followed by (5 t + 1) mod vocab, three quarters of the time; one position in eight is padding."""
    t = torch.randint(1, vocab, (tokens,), generator=generator, device="cuda")
    after = torch.where(torch.rand(tokens, generator=generator, device="cuda") < 0.75, (5 * t + 1) % vocab,
                        torch.randint(vocab, (tokens,), generator=generator, device="cuda"))
    pad = torch.rand(tokens, generator=generator, device="cuda") < 0.125
    targets = torch.where(pad, IGNORE, after)
    weights = (~pad).float() / (~pad).sum()
    return torch.where(pad, PADDING, t), targets, weights


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    model = TiedLm(a.vocab, a.width, a.tokens)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for i in range(a.steps):
        model.step(*batch(a.vocab, a.tokens, g))
        if i % 20 == 0 or i + 1 == a.steps:
            print(f"step {i:4d}  loss {float(model.loss.sum()):.4f}", flush=True)
    assert int(model.status.item()) == 0


if __name__ == "__main__":
    main()
