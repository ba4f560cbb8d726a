"""LMT_FP32_SUMS at the C entry points and in the extension module, without a GPU."""
import pytest

from paper_2402_02447_amd import lmt
from test_lmt_calls import ARG, BF, E4, U8, Tensor, embed, grad, loss, matmul, module, quantize  # noqa: F401


def test_the_flag_is_the_products_alone():
    L = lmt._lib()
    assert matmul(L, m=0, flags=4) == 0 and matmul(L, m=0, flags=5) == 0
    for flags in (2, 6, 8, 12):
        assert matmul(L, flags=flags) == ARG
    assert grad(L, flags=4) == ARG and quantize(L, flags=4) == ARG


def test_the_extension_module_hands_it_on(module):  # noqa: F811
    args = [Tensor((3, 640), E4, 0x10), Tensor((3, 8), U8, 0x20), Tensor((9, 640), E4, 0x30), Tensor((9, 8), U8, 0x40), Tensor((3, 9), BF, 0x60), None]
    for accumulate in (False, True):
        for more, flag in (((), 0), ((False,), 0), ((True,), 4)):
            rc, seen = module("matmul", *args, accumulate, 5, *more)
            assert rc == 7 and seen[12] == accumulate + flag and seen[-1] == 5
    with pytest.raises(TypeError):
        module("matmul", *args, False, 5, True, True)
