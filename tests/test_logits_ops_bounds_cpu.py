"""Further refusals of the calls on logits in memory and on 8-bit matrices, made on the host before any CUDA call
(the addresses are never dereferenced)."""
import ctypes
import itertools

import pytest

from paper_2602_19362_b200 import binding as B, build

OUT, ST = ctypes.c_void_p(0x2000), ctypes.c_void_p(0)
INVALID = -1


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def test_quantize_refuses_scales_that_share_a_place(L):
    """Every layout of 1 to 4 by 1 to 4 scales with strides up to 6, against a count of the places.  A call that is not
    refused for its scales is refused for the alignment of x, which is looked at last."""
    for nr, nc, sr, sc in itertools.product(range(1, 5), range(1, 5), range(7), range(7)):
        apart = len({i * sr + j * sc for i in range(nr) for j in range(nc)}) == nr * nc
        for b in (1, 128):
            rows, cols = (nr if b == 1 else 128 * nr - 5), 128 * nc - 1
            m = B.OaplScaled(0x1000, 0x2000, rows, cols, 1024, sr, sc, 3, b)
            rc = L.oapl_quantize(ctypes.c_void_p(0x2001), 0, rows, cols, 2000, m, 0, ST)
            assert rc == (-2 if apart else INVALID), (nr, nc, sr, sc, b)
            rc = L.oapl_quantize(ctypes.c_void_p(0x2001), 0, cols, rows, 2000, m, B.OAPL_QUANT_TRANSPOSE, ST)
            assert rc == (-2 if apart else INVALID), (nr, nc, sr, sc, b)


def test_scales_of_operands_may_share_a_place(L):
    # one scale for all rows of a column block is a legal operand: refused here only for C's alignment
    m = B.OaplScaled(0x1000, 0x2000, 256, 512, 512, 0, 1, 3, 1)
    assert L.oapl_scaled_matmul(m, m, ctypes.c_void_p(0x2001), 0, 256, 0, None, ST) == -2


@pytest.mark.parametrize("off, ld_d", [(2, 2100), (-2, 2100), (1000, 2100), (1998, 2100), (-1998, 2100), (2 * 2100 + 500, 2100),
                                       (-2 * 2100 * 7 - 4, 2100), (2 * 2100 * 63 + 1998, 2100), (2 * 2100 - 1000, 2100),
                                       (4000, 2099), (-4000, 2101), (2, 1 << 40)])
def test_gradient_refuses_a_place_that_overlaps_the_logits(L, off, ld_d):
    """64 rows of 1000 bf16 logits, 2100 elements apart: bytes that a row of the result shares with any row of them."""
    p = B.OaplLogits(0x100000, 64, 2100, 1000, 0, 0x3000, 0x4000, 1.0)
    d = ctypes.c_void_p(p.logits + off)
    assert L.oapl_logits_logprobs_bwd(p, OUT, OUT, OUT, OUT, 0, None, None, d, ld_d, ST) == INVALID


def test_debug_product_arguments(L):
    f = L.oapl_debug_scaled_matmul
    m = B.OaplScaled(0x1000, 0x2000, 256, 512, 512, 1, 256, 3, 1)
    off = ctypes.c_void_p(0x2001)           # off C's alignment: nothing is launched in any case
    assert f(m, m, off, 0, 256, 0, OUT, 0, 0, ST) == -2
    assert f(m, m, off, 0, 256, 0, OUT, 1000, 3, ST) == -2
    for status, cycles, step in [(None, 0, 0), (OUT, -1, 0), (OUT, 0, -1), (OUT, 0, 1), (OUT, 100_000_001, 1),
                                 (OUT, 4_000_000_001, 0)]:
        assert f(m, m, off, 0, 256, 0, status, cycles, step, ST) == INVALID
