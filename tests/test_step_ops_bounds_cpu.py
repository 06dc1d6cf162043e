"""The ends of what the host sides of the embedding, the residual norm, the gradient norm and clipping take."""
import ctypes

import pytest

from paper_2602_19362_b200 import binding as B, build

ST = ctypes.c_void_p(0)
INVALID, MISALIGNED = -1, -2


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def test_clipping_by_the_norm_checks_its_arguments(L):
    gb = 1 << 36
    t = (B.OaplTensor * 2)(B.OaplTensor(gb, 2 * gb, 1000, 0, 0), B.OaplTensor(3 * gb, 4 * gb, 1000, 0, 0))
    f = lambda t=t, c=2, s=1.0, sq=5 * gb, norm=6 * gb, clip=1.0: L.oapl_grad_clip_ex(t, c, s, sq, norm, clip, ST)  # noqa: E731
    assert f(t=None) == f(c=0) == f(s=float("nan")) == f(sq=None, norm=None) == f(clip=0.0) == f(clip=float("inf")) == INVALID
    assert f(norm=6 * gb + 2) == f(sq=None, norm=6 * gb + 1) == f(sq=5 * gb + 2) == MISALIGNED
    t[1].out = 3 * gb + 2
    assert f() == INVALID
    with pytest.raises(TypeError):
        B.oapl_grad_clip(type("List", (), dict(device=0, array=t, count=2))(), None, 1.0)
