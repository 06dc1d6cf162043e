"""oapl_logits_logprobs and its gradient where order, magnitude or cancellation decide: ids that repeat the target,
peaked rows, rows whose log-sum-exp is too large for its digits to say anything of a probability."""
import math

import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24      # half a step of fp32


def forward(z, targets, mask=None, scale=1.0):
    """lse and entropy as the forward leaves them."""
    N = z.shape[0]
    L = B.make_logits(z, targets, mask, scale)
    lp, ent, lse = (torch.empty(N, device="cuda") for _ in range(3))
    B.oapl_logits_logprobs(L, lp, ent, lse)
    return L, lp, ent, lse


@pytest.mark.parametrize("K", [2, 3, 32])
@pytest.mark.parametrize("N", [3, 900])
def test_gradient_of_a_target_repeated_among_the_ids_has_one_order(N, K):
    V = 1000
    g = torch.Generator(device="cuda").manual_seed(K)
    z = torch.randn(N, V, device="cuda", generator=g)
    targets = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
    # p of the target is 0, so the entry is the sum of its point terms, bit for bit
    z.scatter_(1, targets.long()[:, None], -math.inf)
    ids = targets[:, None].repeat(1, K).contiguous()
    gl, gt = torch.randn(N, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g)
    gl[0], gt[0] = 1.0, 2.0 ** -24          # 1 from the left, 1 + K 2^-24 when the small ones are added first
    gl[1], gt[1] = 2.0 ** -24, 1.0
    want = gl.clone()
    for k in range(K):
        want = want + gt[:, k]              # the target's term first, then by k
    L, _, ent, lse = forward(z, targets)
    first = None
    for _ in range(8):
        d = torch.empty_like(z)
        B.oapl_logits_logprobs_bwd(L, lse, ent, gl, None, gt, ids, d)
        assert torch.equal(d.gather(1, targets.long()[:, None])[:, 0], want)
        first = d if first is None else first
        assert torch.equal(d, first)
    B.oapl_logits_logprobs_bwd(L, lse, ent, gl, None, gt, ids, z)      # over the logits
    assert torch.equal(z, first)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V,N", [(40000, 14), (152064, 14), (40000, 840)])
def test_entropy_of_peaked_rows(t, V, N):
    # Two logits b bits apart, the smaller one first in the same thread's part of the row, so that the reference
    # of the sums is up to 8 bits below the maximum; everything else is -inf, whose terms are exact zeros.
    bits = torch.tensor([0.5, 1, 3, 5, 7.5, 7.9, 8.2, 9, 12, 16, 20, 24, 30, 40], device="cuda")
    z = torch.full((14, V), -math.inf, device="cuda")
    z[:, 0] = 3.3
    z[:, V - V % 2048 - 2048] = 3.3 + bits * math.log(2)
    z = z.to(TYPES[t]).repeat(N // 14, 1)
    two = z[:, [0, V - V % 2048 - 2048]].double()
    lp = torch.log_softmax(two, 1)
    want = -(lp.exp() * lp).sum(1)
    # k: how far the reference may trail.  ln S: the exponential's 2^-22, one sum, a logarithm of at most k ln 2 with
    # two roundings.  ln 2 T / S, at most k ln 2: two roundings of T, one of S, the quotient's, the product's and
    # ln 2's.  ln p of the smaller logit: 2 b U + 2^-22, times p (b + 1), below 7 U.
    b = (two[:, 1] - two[:, 0]) / math.log(2)
    k = torch.where(b < 8.1, b, 0.0)
    tol = (12 + 8 * k) * U
    for K in (0, 8):
        ent = torch.empty(N, device="cuda")
        top = torch.empty(N, K, device="cuda") if K else None
        B.oapl_logits_logprobs(B.make_logits(z), None, ent, None, top)
        assert bool(((ent.double() - want).abs() <= tol).all()), (ent, want)


def exact_gradient(z, targets, gl, ge, gt, ids, scale):
    """From the logits alone, in 64 bits: ln p relative to the row's maximum.  Also the size that roundings scale with."""
    x = z.double()
    d = scale * (x - x.amax(1, keepdim=True))
    lp = torch.log_softmax(d, 1)
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    H = -plp.sum(1, keepdim=True)
    G = gl.double() + gt.double().sum(1)
    point = torch.zeros_like(x).scatter_add_(1, targets.long()[:, None], gl.double()[:, None])
    point.scatter_add_(1, ids.long(), gt.double())
    out = scale * (-(p * G[:, None] + ge.double()[:, None] * (plp + p * H)) + point)
    terms = torch.zeros_like(x).scatter_add_(1, targets.long()[:, None], gl.double().abs()[:, None])
    terms.scatter_add_(1, ids.long(), gt.double().abs())
    size = scale * (p * (gl.double().abs() + gt.double().abs().sum(1))[:, None] + ge.double().abs()[:, None] * (plp.abs() + p * H + p))
    dist = torch.where(p > 0, d.abs(), torch.zeros_like(d))
    return out, size, dist, scale * terms


@pytest.mark.parametrize("t,low", [("bf16", -1e9), ("f32", -1e9), ("f32", -1e20), ("bf16", -1e20), ("f16", -65504.0),
                                   ("bf16", -3000.0), ("f32", 1e9), ("f32", 1e5), ("bf16", 4e4), ("f16", 6e4)])
@pytest.mark.parametrize("scale,N,V", [(1.0, 6, 3001), (1 / 0.7, 700, 3001), (1.3, 6, 152064), (1 / 0.7, 60, 50021),
                                       (1.0, 1200, 70001)])
def test_gradient_of_rows_with_a_large_offset(t, low, scale, N, V):
    g = torch.Generator(device="cuda").manual_seed(V)
    kinds = 6
    z = torch.randn(kinds, V, device="cuda", generator=g)
    z[0] = low                                    # nothing but a finite mask value, or the offset alone: uniform
    z[1] = low
    z[1, ::2] = -math.inf                         # some excluded altogether
    z[2] = low + z[2] * abs(low) * 2.0 ** -6      # an offset, and logits as far apart as the type tells them
    z[3] = low
    z[3, V // 2] = low + abs(low) / 8             # one above the rest
    if t == "f16":
        z[2:4].clamp_(-65504.0, 65504.0)
    z = z.to(TYPES[t]).repeat(-(-N // kinds), 1)[:N].contiguous()      # rows 4, 5: ordinary ones beside them
    targets = torch.full((N,), 1, dtype=torch.int32, device="cuda")
    targets[0] = V - 1
    gl, ge = torch.randn(N, device="cuda", generator=g), torch.randn(N, device="cuda", generator=g)
    gt = torch.rand(N, 3, device="cuda", generator=g)
    ids = torch.tensor([[1, V // 2, V - 1]], dtype=torch.int32, device="cuda").repeat(N, 1)
    L, _, ent, lse = forward(z, targets, None, scale)
    d = torch.empty(N, V + 3, dtype=z.dtype, device="cuda")[:, :V]
    B.oapl_logits_logprobs_bwd(L, lse, ent, gl, ge, gt, ids, d)
    want, size, dist, point = exact_gradient(z, targets, gl, ge, gt, ids, scale)
    fi = torch.finfo(z.dtype)
    # One rounding to the type.  p: 2^-22 of the exponential; ln p: behind an lse of up to 1024 its half step 2^-15 and
    # its product with ln 2, 2^-14; otherwise ln S as a sum of V / 128 terms a thread and a tree of 13; and five
    # roundings of a distance (scale, difference, multiply-add, two of the change of base).  The forward's entropy: its
    # two sums of as many terms.  The rest: roundings of factors and terms.
    rel = 2.0 ** -22 + 2.0 ** -13 + (5 * dist + V / 128 + 100) * U
    tol = fi.eps / 2 * want.abs() + size * rel * (1 + fi.eps) + 12 * U * point + fi.smallest_normal * fi.eps + 1e-35
    bad = ~((d.double() - want).abs() <= tol)
    assert not bool(bad.any()), (bad.nonzero()[:4], d[bad][:4], want[bad][:4], tol[bad][:4])
    again = z.clone()
    L2 = B.make_logits(again, targets, None, scale)
    B.oapl_logits_logprobs_bwd(L2, lse, ent, gl, ge, gt, ids, again)       # over the logits
    assert torch.equal(again, d)


def test_gradient_of_a_row_that_does_not_belong_to_its_lse_is_bounded():
    # no finite logit, but an lse that says otherwise: p is 0, the point term is left
    z = torch.full((2, 700), -math.inf, device="cuda")
    targets = torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    d = torch.empty_like(z)
    B.oapl_logits_logprobs_bwd(B.make_logits(z, targets), torch.tensor([2e3, -5e9], device="cuda"), None,
                               torch.ones(2, device="cuda"), None, None, None, d)
    want = torch.zeros_like(z).scatter_(1, targets.long()[:, None], 1.0)
    assert torch.equal(d, want)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("first", [True, False])
def test_gradient_between_the_rows_of_the_logits(t, first):
    # [logits | gradient] or [gradient | logits] in one buffer, rows side by side
    N, V = 70, 5003
    g = torch.Generator(device="cuda").manual_seed(1)
    buf = torch.randn(N, 2 * V, device="cuda", generator=g).to(TYPES[t])
    z, d = (buf[:, :V], buf[:, V:]) if first else (buf[:, V:], buf[:, :V])
    targets = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
    gl = torch.randn(N, device="cuda", generator=g)
    old = z.clone()
    L, _, ent, lse = forward(z, targets)
    B.oapl_logits_logprobs_bwd(L, lse, ent, gl, gl, None, None, d)
    assert torch.equal(z, old)
    want = torch.empty_like(old)
    B.oapl_logits_logprobs_bwd(B.make_logits(old, targets), lse, ent, gl, gl, None, None, want)
    assert torch.equal(d, want)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("N,K", [(3, 0), (3, 7), (700, 0), (700, 7)])
@pytest.mark.parametrize("offset", [0.0, 1e8])
def test_forward_sums_of_every_variant(t, N, K, offset):
    """CTAs of 256 and of 128 threads, whole rows and split ones, and (with the offset) the careful pass over a row."""
    V = 50021
    g = torch.Generator(device="cuda").manual_seed(N + K)
    z = (torch.randn(N, V, device="cuda", generator=g) * 3).to(TYPES[t])
    if offset:
        step = offset * torch.finfo(z.dtype).eps          # neighbouring numbers of the type beside the offset
        z = (offset + (z.float() / 4).round().double() * step).to(TYPES[t])
    targets = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
    scale = 1.0 if not offset else 0.7 / step
    top = torch.empty(N, K, device="cuda") if K else None
    lp, ent = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    B.oapl_logits_logprobs(B.make_logits(z, targets, None, scale), lp, ent, None, top)
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    x = s32 * (z.double() - z.double().amax(1, keepdim=True))
    ln_p = torch.log_softmax(x, 1)
    p = ln_p.exp()
    want, mean = -(p * ln_p).sum(1), -(p * x).sum(1)
    at = x.gather(1, targets.long()[:, None])[:, 0].abs()
    # A running sum takes at most V / 128 terms (128 threads, one lane per sum: the careful pass and narrow CTAs bound all
    # others), then a tree of 13; 2^-22 of the exponential; x: a multiply-add or a difference and a product, the
    # factor's own rounding, at a distance of `mean` on average.  ln p of the target: its distance and ln S likewise.
    rel = (V / 128 + 13) * U + 2.0 ** -22 + 4 * U * (mean + 1)
    assert bool(((ent.double() - want).abs() <= (2 * rel + 8 * U) * (mean + 1)).all())
    got = ln_p.gather(1, targets.long()[:, None])[:, 0]
    assert bool(((lp.double() - got).abs() <= rel + 4 * U * (at + got.abs() + 8)).all())
    if K:
        best = ln_p.sort(1, descending=True).values[:, :K]
        assert bool(((top.double() - best).abs() <= (rel + 4 * U * (best.abs().amax(1) + 8))[:, None]).all())
