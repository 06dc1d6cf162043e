"""oapl_scaled_matmul when a pipeline wait runs out: the status word, NaN in what was not computed, and a context that
stays usable."""
import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TIMEOUT = -8


def operands(M, N, K, bb):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    A, W = B.alloc_scaled(M, K, 1), B.alloc_scaled(N, K, bb)
    B.oapl_quantize(torch.randn(M, K, device="cuda", generator=g), A)
    B.oapl_quantize(torch.randn(N, K, device="cuda", generator=g), W)
    return A, W


# columns up to 16, 32 and 64 rows of A; pairs with one tile each; pairs with several, whose first ones are done when
# the step that is left out comes (16 K blocks a tile)
@pytest.mark.parametrize("M,N,K,step", [(3, 700, 1100, 1), (20, 5000, 2048, 2), (64, 40000, 1024, 6), (200, 300, 900, 5),
                                        (2600, 4000, 2048, 20)])
@pytest.mark.parametrize("out,pad,accumulate", [("bf16", 0, False), ("f32", 0, True), ("f16", 3, False), ("f32", 5, True)])
@pytest.mark.parametrize("bb", [128, 1])
def test_a_wait_that_runs_out_shows(M, N, K, step, out, pad, accumulate, bb):
    A, W = operands(M, N, K, bb)
    start = torch.full((M, N + pad), 2.0, dtype=TYPES[out], device="cuda")
    want, st = start.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_scaled_matmul(A, W, want[:, :N], accumulate, st)
    assert int(st) == 0 and not bool(torch.isnan(want).any())
    C = start.clone()
    B.oapl_debug_scaled_matmul(A, W, C[:, :N], st, accumulate, wait_cycles=2_000_000, skip_step=step)
    torch.cuda.synchronize()
    assert int(st) == TIMEOUT
    # every element is the product's or NaN; nothing else is written
    lost = torch.isnan(C[:, :N])
    assert bool(lost.any()) and torch.equal(torch.where(lost, want[:, :N], C[:, :N]), want[:, :N])
    assert torch.equal(C[:, N:], start[:, N:])
    if step * 128 * (4 if M <= 16 else 2 if M <= 64 else 1) <= K:
        assert bool(lost.all())              # the step belongs to every CTA's first tile
    # a healthy launch afterwards, under a short limit too
    st.zero_()
    C = start.clone()
    B.oapl_debug_scaled_matmul(A, W, C[:, :N], st, accumulate, wait_cycles=50_000_000)
    assert int(st) == 0 and torch.equal(C, want)
    C = start.clone()
    B.oapl_scaled_matmul(A, W, C[:, :N], accumulate)
    assert torch.equal(C, want)
