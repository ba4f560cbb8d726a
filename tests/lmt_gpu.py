"""Helpers of the GPU tests of lmt.h: matrices that start anywhere in a buffer whose other bytes are watched."""
from __future__ import annotations

import numpy as np
import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64,
      "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "u8": torch.uint8}


class Mat:
    """A rows x cols view with row stride cols + gap, `offset` elements into a buffer of one repeated byte."""

    def __init__(self, rows, cols, kind, gap=0, offset=0, values=None):
        ld, self.size = cols + gap, torch.empty(0, dtype=DT[kind]).element_size()
        n = offset + rows * ld + 8
        self.buffer = torch.full((n * self.size,), 0x5A, dtype=torch.uint8, device="cuda")
        flat = self.buffer.view(DT[kind])
        self.view = flat[offset:offset + rows * ld].view(rows, ld)[:, :cols] if rows else flat[:0].view(0, cols)
        self.rows, self.cols, self.ld, self.offset = rows, cols, ld, offset
        if values is not None:
            self.view.copy_(torch.as_tensor(values))

    def numpy(self):
        return self.view.double().cpu().numpy()

    def untouched_outside(self):
        b = self.buffer.cpu().numpy().reshape(-1, self.size)
        inside = np.zeros(len(b), bool)
        for r in range(self.rows):
            inside[self.offset + r * self.ld:self.offset + r * self.ld + self.cols] = True
        return bool((b[~inside] == 0x5A).all())


def typed(x, kind):
    """x rounded to a type, as float64."""
    return torch.as_tensor(np.asarray(x, np.float64)).to(DT[kind]).double().numpy()


def within(got, want, bound):
    """Every element within its bound; infinities and NaN where they are wanted."""
    got, want, bound = (np.asarray(a, np.float64) for a in (got, want, bound))
    assert got.shape == want.shape, (got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), "infinities or NaN elsewhere"
    assert np.isfinite(got[fine]).all(), "infinities or NaN where there are none"
    over = np.abs(got[fine] - want[fine]) - bound[fine]
    assert over.size == 0 or over.max() <= 0, f"{int((over > 0).sum())} of {over.size} out of bounds, worst by {over.max():.3e}"
