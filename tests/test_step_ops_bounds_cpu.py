"""The ends of what the host sides of the embedding, the residual norm, the gradient norm and clipping take."""
import ctypes
import re
import subprocess

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


def test_the_library_holds_the_residual_kernels_that_calls_reach_and_no_others(L):
    names = subprocess.run(["nm", "-C", "--defined-only", build.LIB], capture_output=True, text=True, check=True).stdout
    have = set(re.findall(r"oapl::residual_(fwd|bwd)_kernel<(\w+), (\d+), (\d+), (\w+), (\d+), (\w+), (\d+)>", names))
    anything, post, plain, post_full, full = range(5)
    want = set()
    for t, ke in (("__nv_bfloat16", 8), ("__half", 8), ("float", 4)):
        # elements a thread, whether a row is a warp's, threads at most
        for e, warp, threads in ((8, True, 256), (16, True, 256), (8, False, 256), (16, False, 256), (16, False, 512), (32, False, 512)):
            for level in (True, False):
                if t == "float" and e == 32 and level:
                    continue        # fp32 rows as wide as these are read where they are
                forms = {anything}
                forms |= {post, post_full} if e < 32 or level else set()
                forms |= {plain, full} if e < 32 and level else set()
                shape = (t, str(ke), str(e // ke), str(warp).lower(), str(threads), str(level).lower())
                want |= {("bwd", *shape, str(f)) for f in forms} | {("fwd", *shape, str(f)) for f in (anything, post)}
    assert have == want, (sorted(have - want)[:5], sorted(want - have)[:5])


def test_workspace_of_the_longest_list(L):
    w = L.oapl_grad_norm_workspace_bytes
    one = w(1)                                       # a launch's partial sums
    most = 2 ** 31 - 1
    launches = [n for n in range(950, 970) if w(n) == one][-1]      # tensors of a launch
    for count in (launches + 1, most - launches, most - launches + 1, most - 1, most):
        assert w(count) == one * -(-count // launches), count
