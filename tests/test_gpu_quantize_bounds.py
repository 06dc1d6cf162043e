"""oapl_quantize on values beside the middle between two 8-bit numbers, where the order of roundings shows."""
import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}


def middles(to):
    """The values half way between neighbours of the type, with their neighbours: all positive ones."""
    v = torch.arange(0, 127 if to == "e4m3" else 124, dtype=torch.uint8).view(F8[to]).double()
    assert float(v[-1]) == TOP[to]
    return (v[1:] + v[:-1]) / 2, v[:-1], v[1:]


def near(x, steps=3):
    """Each fp32 number with the `steps` below and above it."""
    bits = x.float().view(torch.int32)[:, None] + torch.arange(-steps, steps + 1, dtype=torch.int32)
    return bits.view(torch.float32)


def quantize(x, to, turn, pow2):
    """Rows of fp32 x in blocks of 1 x 128."""
    out = B.alloc_scaled(*x.shape, 1, F8[to])
    B.oapl_quantize(x.t().contiguous() if turn else x, out, turn, pow2)
    return out.tensors[0].double().cpu(), out.tensors[1].double().cpu()


def rows_of(values, amax):
    """Rows of 128 values whose first one is amax."""
    flat = values.reshape(-1)
    flat = torch.cat([flat, torch.zeros((-len(flat)) % 127)]).view(-1, 127)
    return torch.cat([torch.full((len(flat), 1), amax), flat], 1).float()


@pytest.mark.parametrize("to", ["e4m3", "e5m2"])
@pytest.mark.parametrize("turn", [False, True])
@pytest.mark.parametrize("exp", [-90, -3, 0, 40])
def test_power_of_two_scales_round_once(to, turn, exp):
    # largest magnitude top 2^exp: the scale is 2^exp and x / scale is exact
    m, _, _ = middles(to)
    x = rows_of(near(m) * 2.0 ** exp, TOP[to] * 2.0 ** exp)
    q, s = quantize(x.cuda(), to, turn, True)
    assert bool((s == 2.0 ** exp).all())
    want = (x.double() / 2.0 ** exp).float().to(F8[to]).double()      # exact, then one rounding
    assert torch.equal(q, want)
    q, _ = quantize(-x.cuda(), to, turn, True)
    assert torch.equal(q, -want)


@pytest.mark.parametrize("to", ["e4m3", "e5m2"])
@pytest.mark.parametrize("turn", [False, True])
def test_fp32_inputs_beside_the_middle(to, turn):
    m, lo, hi = middles(to)
    g = torch.Generator().manual_seed(7)
    for amax in [float.fromhex("0x1.3f0abcp+0"), 448.0, 1.0] + torch.rand(12, generator=g).add(0.5).tolist():
        amax = float(torch.tensor(amax))
        x = rows_of(near(m * amax / TOP[to]), amax)
        q, s = quantize(x.cuda(), to, turn, False)
        # the stated rule, each step rounded to fp32 from 64 bits (a quotient of two fp32 numbers that is rounded to
        # 64 bits on the way to 32 is the correctly rounded one: 53 >= 2 * 24 + 2)
        a = (x.double() * 0.875).float().double()
        y = (a / (amax * (0.875 / TOP[to]))).float()
        assert torch.equal(q, y.to(F8[to]).double())
        assert torch.equal(s, torch.full_like(s, amax / TOP[to]).float().double())
        # and one of the two neighbours of the exact quotient, the nearer one outside 2^-23 of the middle
        exact = x.double() * TOP[to] / amax
        at = torch.searchsorted(m, exact.clamp(max=TOP[to]))            # middles below the value
        off = torch.stack([(exact - m[(at - k).clamp(0, len(m) - 1)]).abs() for k in (0, 1)]).amin(0)
        v = torch.cat([lo, hi[-1:]])
        clear = off > 2.0 ** -23 * exact
        assert torch.equal(q[clear], v[at][clear])
        one_of = (q == v[at]) | (q == v[(at - 1).clamp(min=0)]) | (q == v[(at + 1).clamp(max=len(v) - 1)])
        assert bool(one_of.all())


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("to", ["e4m3", "e5m2"])
def test_16_bit_inputs_round_as_the_exact_quotient(t, to):
    # all products of a few block maxima: the quotient in 64 bits, rounded to fp32 and then to 8 bits
    g = torch.Generator().manual_seed(3)
    for amax in [1.0, 1.75, 3.5] + torch.rand(9, generator=g).mul(8).add(0.25).tolist():
        amax = float(torch.tensor(amax, dtype=t))
        x = (torch.rand(60, 127, generator=g) * 2 - 1) * amax
        x = torch.cat([torch.full((60, 1), amax), x], 1).to(t)
        out = B.alloc_scaled(60, 128, 1, F8[to])
        B.oapl_quantize(x.cuda(), out)
        want = (x.double() * TOP[to] / amax).float().to(F8[to]).double()
        assert torch.equal(out.tensors[0].double().cpu(), want)
