"""The embedding's gradient, the residual norm, clipping and the adjustments of logits at the ends of their ranges."""
import math

import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24      # half a step of fp32


def half_step(want, t):
    f = torch.finfo(t)
    return want.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def scratch(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ clipping

def norm_of(tensors):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in tensors))


@pytest.mark.parametrize("t,std", [("f32", 1e25), ("f32", 1e30), ("bf16", 1e30), ("f32", 1.0), ("f32", 1e-30)])
@pytest.mark.parametrize("apart", [False, True])
def test_a_norm_whose_square_leaves_fp32_clips(t, std, apart):
    g = torch.Generator(device="cuda").manual_seed(9)
    tensors = [torch.randn(n, device="cuda", generator=g).mul_(std).to(TYPES[t]) for n in (100, 9000, 3)]
    want = norm_of(tensors)
    outs = [torch.empty(x.numel(), device="cuda") for x in tensors] if apart else None
    before = [x.double() for x in tensors]
    lst = B.make_tensor_list(tensors, outs)
    sq, norm = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_grad_norm(lst, sq, norm, scratch(B.oapl_grad_norm_workspace_bytes(3)), 0.5, st)
    assert int(st) == 0 and math.isinf(float(sq)) == (want > 2e19 * 2)
    B.oapl_grad_clip(lst, sq, 0.25 if std >= 1 else 1e-20, 0.5, norm)
    factor = min(1.0, (0.25 if std >= 1 else float(torch.tensor(1e-20))) / (0.5 * want + 1e-6)) * 0.5
    for b, o in zip(before, outs or tensors):
        w = b * factor
        # 18 half steps of the norm, as where it is formed; the factor's, its product with the scale's and the element's
        assert bool(((o.double() - w).abs() <= half_step(w, o.dtype) + 22 * U * w.abs()).all())


def test_the_norm_decides_where_both_are_given_and_is_enough():
    x = torch.full((1000,), 2.0, device="cuda")
    out = torch.empty_like(x)
    lst = B.make_tensor_list([x], [out])
    four, one = torch.full((1,), 4.0, device="cuda"), torch.full((1,), 1.0, device="cuda")
    for sq in (one, None):
        B.oapl_grad_clip(lst, sq, 1.0, 1.0, four)
        assert bool(((out - 0.5).abs() <= 1e-6).all())
    B.oapl_grad_clip(lst, four, 1.0)
    assert bool(((out - 1.0).abs() <= 2e-6).all())
    # not finite: the factor is the scale
    for bad in (math.inf, math.nan):
        B.oapl_grad_clip(lst, one, 1.0, 0.5, torch.full((1,), bad, device="cuda"))
        assert bool((out == 1.0).all())


def test_a_norm_that_leaves_fp32_is_reported():
    # every element is finite, and so is the sum of their squares in 64 bits
    x = torch.full((1000,), 3e38, device="cuda")
    y = torch.full((1000,), 1e25, device="cuda")
    sq, norm = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    for v, args, status in ((x, (sq, norm), -7), (x, (None, norm), -7), (x, (sq, None), -7),
                            (y, (sq, norm), 0), (y, (None, norm), 0), (y, (sq, None), -7)):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.oapl_grad_norm(B.make_tensor_list([v]), *args, scratch(B.oapl_grad_norm_workspace_bytes(1)), 1.0, st)
        assert int(st) == status, (float(v[0]), args)
