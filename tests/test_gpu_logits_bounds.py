"""oapl_logits_logprobs and its gradient where order, magnitude or cancellation decide: ids that repeat the
target, peaked rows."""
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
