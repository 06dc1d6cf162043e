"""The embedding's gradient, the residual norm, clipping and the adjustments of logits at the ends of their ranges."""
import itertools
import math

import pytest
import torch

from paper_2602_19362_b200 import binding as B
from tests import test_gpu_adjust as adj
from tests import test_gpu_residual as res

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


# ------------------------------------------------------------------------------------------------ residual norm

def residual_scratch(N, d):
    return scratch(B.oapl_residual_norm_workspace_bytes(N, d))


@pytest.mark.parametrize("which", ["pre", "post"])
def test_sums_over_many_rows_stay_near_their_value(which):
    # every row adds c to a column.  A running sum of c beyond 1024 loses nearly 2^-14 of each c, so that one sum over a
    # worker's thousands of rows would be off by hundreds of half steps
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    N, d, c = 3 * 4096 * sms, 520, 1 + 2.0 ** -14 - 2.0 ** -20
    ones, w = torch.ones(N, d, dtype=torch.bfloat16, device="cuda"), torch.ones(d, device="cuda")
    r = torch.full((N,), c, device="cuda")
    got = [torch.zeros(d, device="cuda") for _ in range(2)]
    if which == "pre":
        B.oapl_residual_norm_bwd(B.make_residual(ones, w_pre=w), ones, None, r, ones, None, dw_pre=got[0], ws=residual_scratch(N, d))
        got = got[:1]
    else:
        B.oapl_residual_norm_bwd(B.make_residual(ones, ones, w, w_post=w), None, r, None, None, ones, dgate=got[0], dw_post=got[1],
                                 ws=residual_scratch(N, d))
    # 256 rows in a register, the launches' sums of 256 (one worker per SM at least), 1024 workers in 32 shares and their
    # tree; the terms' and the factors' own roundings
    steps = 256 + N // sms // 256 + 1024 // 32 + 5 + 4
    for g in got:
        off = (g.double() - N * c).abs().max()
        assert float(off) <= steps * U * N * c, float(off) / (U * N * c)


@pytest.mark.parametrize("t,N,d,pad", [("bf16", 1200007, 24, 0), ("f32", 900001, 77, 1), ("f16", 700001, 400, 0), ("bf16", 500001, 401, 2),
                                       ("bf16", 200003, 1112, 0), ("f16", 150001, 1111, 0), ("f32", 60001, 4100, 0),
                                       ("bf16", 60001, 4101, 3), ("bf16", 40003, 9008, 0), ("f32", 20001, 9001, 0)])
@pytest.mark.parametrize("gate", ["none", "row", "column", "full"])
def test_sums_over_many_rows_of_whole_numbers_are_exact(t, N, d, pad, gate):
    g = torch.Generator(device="cuda").manual_seed(d)
    whole = lambda *s, ld=0: torch.randint(-3, 4, (s[0], s[1] + ld) if ld else s, device="cuda", generator=g,  # noqa: E731
                                           dtype=torch.int8).to(TYPES[t])[..., :s[-1]]
    a, b = whole(N, d, ld=pad), whole(N, d, ld=pad)
    w, v = whole(d), whole(d)
    one = torch.ones(N, device="cuda")

    def total(*parts):
        s = torch.zeros(d, dtype=torch.float64, device="cuda")
        for at in range(0, N, 20000):
            x = parts[0][at:at + 20000].double()
            for p in parts[1:]:
                x = x * p[at:at + 20000].double()
            s += x.sum(0)
        return s

    if gate == "none":
        dw = torch.full((d,), 5.0, device="cuda")
        B.oapl_residual_norm_bwd(B.make_residual(a, w_pre=w), a, None, one, b, None, dw_pre=dw, accumulate=True, ws=residual_scratch(N, d))
        assert torch.equal(dw.double(), total(a, b) + 5)
        dw2 = torch.full((d,), 3.0, device="cuda")
        B.oapl_residual_norm_bwd(B.make_residual(a, a, w_pre=w), a, None, one, b, b, dx=torch.empty_like(a), dy=torch.empty_like(a), dw_pre=dw2,
                                 ws=residual_scratch(N, d))
        assert torch.equal(dw2, dw - 5)
    k = {"none": None, "row": whole(N, 1).float(), "column": v, "full": whole(N, d, ld=pad)}[gate]
    dw, dg = torch.empty(d, device="cuda"), torch.empty(d, device="cuda") if gate == "column" else None
    B.oapl_residual_norm_bwd(B.make_residual(a, a, k, w_post=w), None, one, None, None, b, dgate=dg, dw_post=dw, ws=residual_scratch(N, d))
    s = total(a, b, *([k] if gate in ("row", "full") else []))
    assert torch.equal(dw.double(), s * v.double() if gate == "column" else s)
    assert dg is None or torch.equal(dg.double(), s * w.double())


@pytest.mark.parametrize("t,d", [("f32", 1537), ("f32", 7600), ("f32", 9001), ("f32", 12288), ("bf16", 9001), ("bf16", 12288)])
@pytest.mark.parametrize("gate", ["column", "full"])
def test_wide_results_over_inputs(t, d, gate):
    # fp32 rows above 8192 are read where they are, twice, while their results are written
    N = 200
    c = res.make(N, d, t, gate)
    xo, h, rp, rq = [x.clone() for x in res.check_fwd(c)]
    places = ["x", "y"] + (["gate"] if gate == "full" else [])
    for p, q in itertools.permutations(places, 2):
        e = dict(c, **{k: c[k].clone() for k in places})
        rp2, rq2 = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        B.oapl_residual_norm(res.struct(e), e[p], e[q], rp2, rq2)
        assert torch.equal(e[p], xo) and torch.equal(e[q], h) and torch.equal(rp2, rp) and torch.equal(rq2, rq), (p, q)
    dx, dy = torch.empty_like(xo), torch.empty_like(xo)
    dg = torch.empty_like(xo) if gate == "full" else None
    B.oapl_residual_norm_bwd(res.struct(c), xo, rp, rq, c["dh"], c["dxo"], dx, dy, dg)
    places = ["xo", "dh", "dxo", "y"] + (["gate"] if gate == "full" else [])
    for p, q in itertools.permutations(places, 2):
        e = dict(c, xo=xo)
        e = {**e, **{k: e[k].clone() for k in places}}
        dg2 = torch.empty_like(xo) if gate == "full" else None
        B.oapl_residual_norm_bwd(res.struct(e), e["xo"], rp, rq, e["dh"], e["dxo"], e[p], e[q], dg2)
        assert torch.equal(e[p], dx) and torch.equal(e[q], dy), (p, q)
        assert dg is None or torch.equal(dg, dg2)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("d", [72, 256, 1536, 1537, 3584, 5120, 9001])
@pytest.mark.parametrize("alone", [False, True])
def test_gradient_of_the_norm_that_makes_the_heads_rows(t, d, alone):
    # nothing but the head reads x', so dx_out is left out; alone: without a block's result
    N = 300
    c = res.make(N, d, t)
    c["dxo"].zero_()
    if alone:
        c.update(y=None, w_post=None)
    r = res.ref_fwd(c)
    xo = torch.empty_like(c["x"]).copy_(r["xo"])
    rp, rq = (r[k].float() if k in r else None for k in ("rp", "rq"))
    new = lambda: torch.empty_like(c["x"])  # noqa: E731
    dx, dy, dwp, dwq = new(), None if alone else new(), None if alone else torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    B.oapl_residual_norm_bwd(res.struct(c), xo, rp, rq, c["dh"], None, dx, dy, None, dwp, dwq, False, residual_scratch(N, d))
    w = res.ref_bwd(c, xo, rp, rq)
    res.within(dx, w["dx"], w["t_dx"], "dx")
    res.within(dwq, w["dw_pre"], w["t_dw_pre"], "dw_pre")
    if not alone:
        res.within(dy, w["dy"], w["t_dy"], "dy")
        res.within(dwp, w["dw_post"], w["t_dw_post"], "dw_post")


# ------------------------------------------------------------------------------------------------ embedding's gradient

def whole_rows(g, N, d, t="f32"):
    return torch.randint(-8, 9, (N, d), device="cuda", generator=g, dtype=torch.int8).to(TYPES[t])


def check_whole(ids, V, dout, accumulate):
    """Sums of whole numbers are exact in any order, as long as all of them stay below 2^24."""
    N, d = dout.shape
    table = torch.full((V, d), 3.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_embedding_bwd(B.make_lookup(ids, V), dout, table, accumulate, scratch(B.oapl_embedding_workspace_bytes(N, V, d)), st)
    want = torch.full((V, d), 3.0 if accumulate else 0.0, device="cuda").index_add_(0, ids.long(), dout.float())
    assert torch.equal(table, want) and int(st) == 0


# sizes of one launch, of a sort by counting, by digits with the tiles' counts added up by each, and with a launch that
# adds them up; chunks of 32, 32, 32, 64, 128 and 256 positions
@pytest.mark.parametrize("N,chunk", [(1025, 32), (8192, 32), (8193, 32), (40960, 64), (70000, 128), (131073, 256), (300007, 256)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_long_runs_is_exact(N, chunk, accumulate):
    g = torch.Generator(device="cuda").manual_seed(N)
    # one token everywhere, with positive terms: a chunk that is left out shows
    dout = whole_rows(g, N, 24, "bf16").abs()
    check_whole(torch.full((N,), 2, dtype=torch.int32, device="cuda"), 4, dout, accumulate)
    # runs in every alignment to the chunks, in the sorted list; what is left is one run over the rest
    c = chunk
    lens = [c, c, c - 1, 1, c + 1, c - 1, 2 * c, 1, 1, 2 * c - 2, 4 * c, 5, c - 5, c, 1]
    lens += [N - sum(lens)] if N > sum(lens) else []
    ids = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))[:N].to(torch.int32).cuda()
    ids = ids[torch.randperm(N, generator=torch.Generator().manual_seed(3)).cuda()]
    check_whole(ids, len(lens) + 2, dout, accumulate)
    check_whole(ids, len(lens) + 2, whole_rows(g, N, 25, "f16"), accumulate)


@pytest.mark.parametrize("N", [9001, 131072, 131073, 300007])
@pytest.mark.parametrize("V", [1000, 151936, (1 << 20) + 5, 1 << 21])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_large_batches_and_vocabularies_is_exact(N, V, accumulate):
    # one to three passes of digits
    g = torch.Generator(device="cuda").manual_seed(V % 1000 + N)
    u = torch.rand(N, device="cuda", generator=g, dtype=torch.float64)
    ids = ((V ** u).long() - 1).clamp(0, V - 1).to(torch.int32)
    ids[::3] = torch.randint(0, V, (ids[::3].numel(),), device="cuda", generator=g).to(torch.int32)
    ids[5], ids[77] = V - 1, 0
    check_whole(ids, V, whole_rows(g, N, 8, "bf16"), accumulate)


@pytest.mark.parametrize("N", [9001, 140001])
def test_gradient_of_the_largest_vocabulary_is_exact(N):
    V = 2 * 10 ** 9             # four passes of digits, 8 GB
    g = torch.Generator(device="cuda").manual_seed(N)
    ids = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
    ids[::5], ids[1], ids[2] = 1999999999, 0, 1999999998
    check_whole(ids, V, whole_rows(g, N, 1), False)


# ------------------------------------------------------------------------------------------------ adjustments

# slices of 2048, 4096 and 8192 tokens (16384 for the gradient apart) by vectors, of 2048 and 4096 an element at a time;
# more than 512 tokens of a slice change
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("N,V,pad,offset", [(7, 5000, 16, 0), (600, 5001, 16, 0), (700, 8203, 16, 0), (7, 5001, 1, 1), (600, 5000, 1, 1)])
def test_gradient_of_long_histories_over_its_inputs(t, N, V, pad, offset):
    for where in ("z", "d", "apart"):
        c = adj.make(N, V, t, 21, prompt=3000, answer=2500, pad=pad, offset=offset)
        adj.check_bwd(c, torch.tensor([i % 5 != 3 for i in range(N)], dtype=torch.uint8, device="cuda"), where)


def test_biases_before_the_penalties_take_two_calls():
    # the order of some samplers; a token with a bias that changes its sign takes the other branch of the penalty
    N, V = 40, 3001
    c = adj.make(N, V, "f32", 31, allowed=0.8)
    first = {k: c[k] for k in ("bias_start", "bias_id", "bias")}
    rest = {k: v for k, v in c.items() if k not in first}
    count, seen, bias, size, open_ = adj.parts(c)
    mid, out = torch.empty_like(c["z"]), torch.empty_like(c["z"])
    L = B.make_logits(c["z"])
    B.oapl_logits_adjust(L, B.make_adjust(L, **first), mid)
    M = B.make_logits(mid)
    B.oapl_logits_adjust(M, adj.args(M, rest), out)
    r, f, p = (adj.row(c, k, 0.0) for k in ("repetition", "frequency", "presence"))
    z1 = c["z"].double() + bias
    z1 = torch.where(size > 0, mid.double(), z1)        # its rounding decides on the branch where the sum is near zero
    assert bool(((z1 - c["z"].double() - bias).abs() <= 8 * U * (c["z"].double().abs() + size)).all())
    slope = torch.where(seen, torch.where(z1 > 0, 1 / r, r * torch.ones_like(z1)), 1.0)
    want = z1 * slope - f * count - p * (count > 0)
    tol = 4 * U * ((z1 * slope).abs() + (f * count).abs() + (p * (count > 0)).abs()) + half_step(want, torch.float32)
    assert bool(((out.double() - want).abs() <= tol)[open_].all()) and bool((out[~open_] == -math.inf).all())
    d, dz = torch.randn_like(mid), torch.empty_like(mid)
    B.oapl_logits_adjust_bwd(M, adj.args(M, rest), d, dz)
    assert bool(((dz.double() - torch.where(open_, d.double() * slope, 0.0)).abs() <= 4 * U * d.double().abs() * slope).all())
