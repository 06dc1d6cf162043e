"""oapl_grad_norm and oapl_grad_clip against plain 64-bit forms of the same definitions."""
import math

import pytest
import torch

from oracle import oapl_oracle as orc
from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24


def half_step(want, t):
    f = torch.finfo(t)
    return want.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def norm_of(tensors):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in tensors))


def run(tensors, outs, clip, scale=1.0, status=0):
    lst = B.make_tensor_list(tensors, outs)
    ws = torch.full((B.oapl_grad_norm_workspace_bytes(len(tensors)),), 0xFF, dtype=torch.uint8, device="cuda")
    sq, norm = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_grad_norm(lst, sq, norm, ws, scale, st)
    B.oapl_grad_clip(lst, sq, clip, scale)
    assert int(st) == status
    return sq, norm


def check(tensors, outs, clip, scale=1.0):
    scale = torch.tensor(scale, dtype=torch.float32).item()
    before = [t.clone() for t in tensors]
    sq, norm = run(tensors, outs, clip, scale)
    want = norm_of(before) * abs(scale)
    # 32 squares are added in fp32 by a thread (33 half steps of a sum of positive terms), the rest in fp64: half of that
    # for the root, and the results' own rounding
    assert abs(float(norm) - want) <= 18 * U * want + 1e-45
    if 1e-18 < want < 1e18:
        assert abs(float(sq) - want * want) <= 35 * U * want * want
    factor = min(1.0, clip / (want + 1e-6)) * scale
    for b, o in zip(before, tensors if outs is None else outs):
        w = b.double() * factor
        # the norm's share, and roundings of the factor, of its product with the scale and of the element's
        assert bool(((o.double() - w).abs() <= half_step(w, o.dtype) + 22 * U * w.abs()).all())
    if outs is not None:
        assert all(torch.equal(a, b) for a, b in zip(before, tensors))


def make(sizes, t, seed, offset=0, std=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n + offset, device="cuda", generator=g).mul_(std).to(TYPES[t])[offset:] for n in sizes]


SIZES = [1, 7, 8, 0, 255, 8191, 8192, 8193, 16385, 100003, 3, 1 << 20]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("to", list(TYPES))
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_types_sizes_and_alignment(t, to, offset):
    tensors = make(SIZES, t, offset, offset)
    guard = [torch.full((n + 2 * offset + 16,), 5.0, dtype=TYPES[to], device="cuda") for n in SIZES]
    outs = [w[offset:offset + n] for w, n in zip(guard, SIZES)]
    full = norm_of(tensors)
    for clip, scale in [(0.3 * full, 1.0), (10 * full, 1.0), (0.05 * full, 0.125)]:
        check(tensors, outs, clip, scale)
    for w, n in zip(guard, SIZES):
        assert bool((w[:offset] == 5).all()) and bool((w[offset + n:] == 5).all())
    check([x.clone() for x in tensors], None, 0.5 * full, 3.0)      # in place


@pytest.mark.parametrize("count", [1, 480, 481, 959, 960, 961, 2100])
def test_lists_longer_than_a_launch(count):
    sizes = [1 + (i * 37) % 900 for i in range(count)]
    tensors = make(sizes, "f32", count)
    check(tensors, [torch.empty(n, device="cuda") for n in sizes], 0.5 * norm_of(tensors))
    mixed = [x.to(TYPES[["bf16", "f16", "f32"][i % 3]]) for i, x in enumerate(tensors)]
    check(mixed, [torch.empty(n, device="cuda") for n in sizes], 0.5 * norm_of(mixed))
    check(mixed, None, 0.25 * norm_of(mixed))


def test_matrices_and_one_large_tensor():
    g = torch.Generator(device="cuda").manual_seed(2)
    tensors = [torch.randn(1999, 3001, device="cuda", generator=g), torch.randn(64, 3, 5, device="cuda", generator=g).bfloat16()]
    check(tensors, [torch.empty_like(x) for x in tensors], 2.0)
    big = torch.empty((1 << 31) + 4099, dtype=torch.bfloat16, device="cuda").fill_(2.0)     # elements past 32 bits
    sq, norm = run([big], None, 1.0)
    assert float(norm) == pytest.approx(2.0 * math.sqrt(big.numel()), rel=1e-6)
    want = 2.0 / (2.0 * math.sqrt(big.numel()) + 1e-6)
    ends = torch.cat([big[:5000], big[-9000:], big[(1 << 30) - 5:(1 << 30) + 5]])
    assert bool(((ends.double() - want).abs() <= want * 2.0 ** -8).all())


def test_a_norm_below_the_limit_changes_no_bit():
    tensors = make(SIZES, "bf16", 4)
    before = [x.clone() for x in tensors]
    run(tensors, None, 1e6)
    assert all(torch.equal(a, b) for a, b in zip(tensors, before))


@pytest.mark.parametrize("t,std", [("f32", 1e25), ("f32", 1e-30), ("f32", 1e18), ("f32", 1e-13), ("bf16", 1e30), ("bf16", 1e-38)])
def test_values_whose_squares_leave_the_range_of_fp32(t, std):
    tensors = make([100, 9000, 3], t, 9, std=std)
    tensors.append(torch.zeros(5000, dtype=TYPES[t], device="cuda"))
    sq, norm = run(tensors, [torch.empty_like(x) for x in tensors], 1.0)
    want = norm_of(tensors)
    assert abs(float(norm) - want) <= 18 * U * want + 2e-45
    # large and small values in one thread's share
    both = torch.full((8192,), 1e-25, device="cuda")
    both[4000] = 1e22
    _, norm = run([both], [torch.empty_like(both)], 1.0)
    assert float(norm) == pytest.approx(1e22, rel=1e-6)


def test_zeros_infinity_and_nan():
    z = [torch.zeros(9000, device="cuda"), torch.zeros(3, device="cuda").half()]
    check(z, [torch.empty_like(x) for x in z], 1.0)
    for bad in (math.inf, -math.inf, math.nan):
        x = torch.ones(10000, device="cuda")
        x[9999] = bad
        out = torch.empty_like(x)
        sq, norm = run([x], [out], 1.0, 0.5, status=-7)
        assert not math.isfinite(float(norm))
        # not clipped: the caller leaves out the step
        assert torch.equal(out.view(torch.int32), (x * 0.5).view(torch.int32))


def test_only_one_result_and_lists_of_empty_tensors():
    x = torch.full((100,), 2.0, device="cuda")
    lst = B.make_tensor_list([x])
    ws = torch.empty(B.oapl_grad_norm_workspace_bytes(1), dtype=torch.uint8, device="cuda")
    a, b = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    B.oapl_grad_norm(lst, a, None, ws)
    B.oapl_grad_norm(lst, None, b, ws)
    assert float(a) == 400.0 and float(b) == 20.0
    e = B.make_tensor_list([torch.empty(0, device="cuda"), torch.empty(0, device="cuda").half()])
    ws = torch.empty(B.oapl_grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    B.oapl_grad_norm(e, a, b, ws)
    B.oapl_grad_clip(e, a, 1.0)
    assert float(a) == 0.0 and float(b) == 0.0


def test_repeats_bit_for_bit_on_another_stream_and_captured():
    tensors = make(SIZES, "bf16", 12)
    outs = [torch.empty(x.numel(), device="cuda") for x in tensors]
    lst = B.make_tensor_list(tensors, outs)
    ws = torch.empty(B.oapl_grad_norm_workspace_bytes(len(tensors)), dtype=torch.uint8, device="cuda")
    sq, norm = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    call = lambda: (B.oapl_grad_norm(lst, sq, norm, ws, 0.5), B.oapl_grad_clip(lst, sq, 0.1, 0.5))  # noqa: E731
    call()
    want, first = [o.clone() for o in outs], norm.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
        for _ in range(3):
            norm.zero_()
            [o.zero_() for o in outs]
            graph.replay()
    side.synchronize()
    assert torch.equal(norm, first) and all(torch.equal(a, b) for a, b in zip(outs, want))


def test_serves_the_optimizer_step():
    # the norm over all other parameters, taken into the step of the LM-head weight
    g = torch.Generator().manual_seed(3)
    n = 4096
    theta = (0.02 * torch.randn(n, generator=g)).to(torch.bfloat16)
    grad = 1e-2 * torch.randn(n, generator=g)
    rest = make([5000, 77, 1 << 16], "bf16", 21, std=1e-2)
    lst = B.make_tensor_list(rest)
    ws = torch.empty(B.oapl_grad_norm_workspace_bytes(3), dtype=torch.uint8, device="cuda")
    sq = torch.zeros(1, device="cuda")
    B.oapl_grad_norm(lst, sq, None, ws)
    W, master, m, v, gn = theta.clone().cuda(), theta.float().cuda(), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(1, device="cuda")
    hp = [1e-3, 0.9, 0.95, 1e-8, 1e-2, 1.0]
    B.oapl_adamw_step(W, master, grad.cuda(), m, v, 1, *hp, sq, gn)
    lr, b1, b2, eps, wd, clip = (float(torch.tensor(x, dtype=torch.float32)) for x in hp)
    other = norm_of(rest) ** 2
    want = orc.adamw_step(theta.double().numpy(), grad.double().numpy(), 0 * grad.double().numpy(), 0 * grad.double().numpy(), 1,
                          lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, clip_norm=clip, other_sq_norm=other)
    assert float(gn) == pytest.approx(want[3], rel=1e-5)
    assert torch.allclose(m.cpu().double(), torch.from_numpy(want[1]), rtol=1e-5, atol=1e-12)


def test_binding_refusals():
    x = torch.zeros(16, device="cuda")
    for bad in (lambda: B.make_tensor_list([x[::2]]), lambda: B.make_tensor_list([x.double()]),
                lambda: B.make_tensor_list([x], [x[:8]]), lambda: B.make_tensor_list([x, x.cpu()])):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        B.make_tensor_list([x], [x, x])
    lst = B.make_tensor_list([x])
    sq = torch.zeros(1, device="cuda")
    with pytest.raises(B.OaplError, match="WORKSPACE_TOO_SMALL"):
        B.oapl_grad_norm(lst, sq, None, torch.zeros(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_grad_clip(lst, sq, 0.0)
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_grad_clip(B.make_tensor_list([x[:8]], [x[4:12]]), sq, 1.0)
