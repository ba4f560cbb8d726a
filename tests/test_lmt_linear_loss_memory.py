"""What the loss of a product keeps instead of the logits: the size of its workspace, without a GPU."""
import pytest
import torch

import fake_device
from paper_2402_02447_amd import lmt
from test_lmt_attention_calls import LIB

F16, BF = torch.float16, torch.bfloat16
MANY = [(16384, 30522, 1024), (65536, 30522, 2048), (131072, 30522, 1024), (131072, 130000, 1024), (1 << 20, 30522, 768), (8192, 1 << 20, 256), (300, 1 << 22, 64)]


@pytest.mark.parametrize("dtype,sizes", [(t, s) for t in (F16, BF) for s in MANY] + [(BF, (8192, 30522, 1024))])
def test_the_workspace_is_less_than_16_bit_logits(dtype, sizes):
    rows, classes, _ = sizes
    assert lmt.linear_cross_entropy_workspace(*sizes, dtype=dtype) < 2 * rows * classes
    assert lmt.linear_cross_entropy_workspace(*sizes, False, dtype) < rows * classes


def up(x, by):
    return -(-x // by) * by


@pytest.mark.parametrize("rows", [1, 64, 256, 257, 2432, 8192, 50000, 1 << 18])
@pytest.mark.parametrize("classes", [7, 2003, 30522, 250_001])
@pytest.mark.parametrize("width", [64, 257, 1024])
def test_the_workspace_does_not_grow_with_the_logits(rows, classes, width):
    """A piece of g (2^27 elements or one block of 256 classes, whole blocks of 64 rows) in two forms for fp16 and as often again for up to 256 rows; copies of x (two) and the table by whole blocks
    of 64; at most 16 parts of each gradient in fp32; a maximum and a sum for each row and 128 classes, 24 bytes a row."""
    piece = up(min(classes, (1 << 27) // rows + 1), 256)
    for dtype, forms in ((BF, 1), (F16, 2), (None, 2)):
        most = 2 * up(rows, 64) * piece * forms * (2 if rows <= 256 else 1) + 2 * up(width, 64) * (2 * rows + classes) + 4 * 16 * width * (rows + piece)
        most += 8 * rows * up(classes, 128) // 128 + 24 * rows + 16 * 256
        assert lmt.linear_cross_entropy_workspace(rows, classes, width, dtype=dtype) <= most


def test_the_size_for_a_type_is_that_of_aligned_calls():
    for sizes in ((100, 500, 64), (5000, 30522, 1024), (300, 2000, 100), (64, 70, 8)):
        any_call = lmt.linear_cross_entropy_workspace(*sizes)
        assert all(0 < lmt.linear_cross_entropy_workspace(*sizes, dtype=t) <= any_call for t in (F16, BF))
    assert lmt.linear_cross_entropy_workspace(100, 500, 64, dtype=BF) < lmt.linear_cross_entropy_workspace(100, 500, 64, dtype=F16)
    assert lmt.linear_cross_entropy_workspace(0, 5, 5, dtype=BF) == lmt.linear_cross_entropy_workspace(5, 1 << 23, 5, dtype=BF) == 0
    with pytest.raises(ValueError, match="dtype"):
        lmt.linear_cross_entropy_workspace(5, 5, 5, dtype=torch.float32)
    assert lmt._lib().lmt_linear_cross_entropy_workspace_of(lmt.LMT_F32, 5, 5, 5, 1) == 0


def test_a_call_takes_what_it_needs_and_refuses_less(tmp_path):
    fake_device.run(fake_device.build(tmp_path), LIB + """
of, any_call = L.lmt_linear_cross_entropy_workspace_of, L.lmt_linear_cross_entropy_workspace
of.restype = c_uint64
def call(dt, rows, classes, width, ws, x=GB, ld=None, table=GB, gx=GB):
    return L.lmt_linear_cross_entropy(P(x), U(ld or width), P(table), U(width), dt, U(rows), U(classes), U(width), P(GB), 6, c_int64(-100), None, P(GB), P(GB), P(gx), U(width), P(gx), dt, U(width), 0, None, P(GB), U(ws), None)
for dt in (1, 2):
    for rows, classes, width in ((100, 500, 64), (300, 3000, 128), (257, 700, 100), (8192, 30522, 1024)):
        for gx in (GB, None):
            size = U(rows), U(classes), U(width), 1 if gx else 0
            exact, most = of(dt, *size), any_call(*size)
            assert call(dt, rows, classes, width, exact, gx=gx) == 0 and call(dt, rows, classes, width, exact - 1, gx=gx) == -6
            for other in (dict(x=GB + 2), dict(ld=width + 1), dict(table=GB + 8)):
                assert call(dt, rows, classes, width, most, gx=gx, **other) == 0
                assert call(dt, rows, classes, width, exact, gx=gx, **other) == (-6 if width % 64 == 0 else 0)
""")
