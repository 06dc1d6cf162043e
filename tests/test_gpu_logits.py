"""oapl_logits_logprobs and its gradient against plain 64-bit forms of the same definitions."""
import math

import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24      # half a step of fp32


def ref_fwd(z, targets, mask, K, scale=1.0):
    """Everything in 64 bits, from the definition; a sort that keeps equal values in order."""
    x = z.double() * scale
    m = x.amax(1, keepdim=True)
    empty = torch.isneginf(m[:, 0])
    m = torch.where(torch.isfinite(m), m, 0.0)
    e = torch.exp(x - m)
    s = e.sum(1)
    lse = m[:, 0] + torch.log(s)
    lp = (x - m) - torch.log(s)[:, None]      # relative to the maximum: a huge common offset costs nothing
    p = torch.exp(lp)
    ent = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    logp = lp.gather(1, targets.long()[:, None])[:, 0]
    live = mask.bool()
    broken = (torch.isnan(x) | (x == math.inf)).any(1)
    nan = torch.full_like(lse, math.nan)
    out = dict(lse=torch.where(broken, nan, torch.where(empty, -math.inf, lse)),
               ent=torch.where(broken, nan, torch.where(empty, 0.0, ent)),
               logp=torch.where(broken, nan, torch.where(empty, -math.inf, logp)))
    # the mean distance below the maximum, in bits: what rounding of the exponents can move
    out["bits"] = torch.nan_to_num((torch.where(p > 0, p * (m - x), torch.zeros_like(p))).sum(1) / math.log(2))
    if K:
        key = torch.where(torch.isnan(z), -math.inf, z.double() + 0.0)
        v, i = torch.sort(key, dim=1, descending=True, stable=True)
        pad = max(0, K - v.shape[1])
        v = torch.nn.functional.pad(v[:, :K], (0, pad), value=-math.inf)
        i = torch.nn.functional.pad(i[:, :K], (0, pad), value=-1)
        none = torch.isneginf(v)
        out["id"] = torch.where(none | ~live[:, None], -1, i)
        tl = torch.where(none, -math.inf, (v * scale - m) - torch.log(s)[:, None])
        out["top"] = torch.where(live[:, None], torch.where(broken[:, None], math.nan, tl), 0.0)
    for k in ("lse", "ent", "logp"):
        out[k] = torch.where(live, out[k], 0.0)
    return out


def close(got, want, tol, what):
    got, want = got.double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bool(bad.any()), (what, got[bad][:5], want[bad][:5], (got - want).abs()[bad][:5])


def check_fwd(z, targets, mask, K, scale=1.0, status=0):
    N, V = z.shape
    dev = z.device
    new = lambda *s: torch.full(s, 7.5, device=dev)
    lp, ent, lse = new(N), new(N), new(N)
    top = new(N, K) if K else None
    ids = torch.full((N, K), -77, dtype=torch.int32, device=dev) if K else None
    st = torch.zeros(1, dtype=torch.int32, device=dev)
    L = B.make_logits(z, targets, mask, scale)
    B.oapl_logits_logprobs(L, lp, ent, lse, top, ids, st)
    assert int(st) == status
    r = ref_fwd(z, targets, mask if mask is not None else torch.ones(N, device=dev), K, scale)
    # A thread adds at most n terms to a running sum (n roundings), then a tree of 13; e^x carries 2^-22 of
    # the exponential and 4 roundings of x (a difference, a factor, a product, the factor's own).
    n = V / 512 + 16
    rel = (n + 13) * U + 2.0 ** -22 + 4 * U * math.log(2) * (r["bits"] + 1)
    t_lse = rel + 4 * U * (r["lse"].abs().nan_to_num(0, 0, 0) + 1)
    z_t = z.gather(1, targets.long().clamp(0, V - 1)[:, None])[:, 0].double().abs().nan_to_num(0, 0, 0) * scale
    t_lp = t_lse + 4 * U * (z_t + 1)
    close(lse, r["lse"], t_lse, "lse")
    close(lp, r["logp"], t_lp, "logp")
    close(ent, r["ent"], (2 * rel + 8 * U) * (r["bits"] + 1), "entropy")
    if K:
        assert torch.equal(ids.long(), r["id"])
        close(top, r["top"], (t_lse + 4 * U * (r["top"].abs().nan_to_num(0, 0, 0).amax(1) + r["lse"].abs().nan_to_num(0, 0, 0) + 1))[:, None], "top")
    return lp, ent, lse, top, ids


def make(N, V, t, seed, offset=0, pad=0, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.randn(N * (V + pad) + offset, device="cuda", generator=g).mul_(spread).to(TYPES[t])
    z = flat[offset:].view(N, V + pad)[:, :V]
    targets = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
    mask = (torch.rand(N, device="cuda", generator=g) < 0.8).to(torch.uint8)
    return z, targets, mask


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 31, 255, 257, 1000, 2049, 8191, 8200, 50021])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5)])
def test_forward_sizes(t, V, offset, pad):
    for N, K in [(1, 8), (3, 1), (37, 20), (33, 0)]:
        z, targets, mask = make(N, V, t, V + N, offset, pad)
        check_fwd(z, targets, mask if N > 1 else None, K)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 19, 40, 80, 160, 400])
def test_forward_rows_split_over_ctas(t, N):
    # one row over eight CTAs down to one CTA per row
    z, targets, _ = make(N, 152064, t, N)
    check_fwd(z, targets, None, 32)
    check_fwd(z, targets, None, 5, scale=1 / 0.7)


@pytest.mark.parametrize("t,V,offset,pad", [("bf16", 9, 1, 2), ("f16", 1024, 0, 0), ("bf16", 4096, 0, 8), ("f16", 12295, 3, 4),
                                            ("f32", 8209, 1, 0), ("bf16", 50021, 0, 2)])
def test_forward_more_rows_than_sms_hold(t, V, offset, pad):
    # narrow CTAs with alternatives, whole batches and a last one, rows on and off 16-byte boundaries
    z, targets, mask = make(1201, V, t, V, offset, pad)
    check_fwd(z, targets, mask, 7)
    check_fwd(z, targets, None, 0)


def test_forward_vocabulary_larger_than_the_kept_group_maxima():
    # more than 32 batches of a thread: a group holds several
    z, targets, _ = make(200, 600011, "bf16", 3)
    check_fwd(z, targets, None, 20)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_forward_order_and_ties(t):
    V = 20011
    up = torch.linspace(-8, 8, V, device="cuda")
    perm = torch.randperm(V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    rows = [up, up.flip(0), torch.zeros(V, device="cuda"), torch.full((V,), -3.0, device="cuda"),
            torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0),        # -0 and 0 are equal
            (up * 2).round(), (up[perm]).round(), torch.where(perm < 12, 5.0, 1.0),
            torch.where(torch.arange(V, device="cuda") >= V - 9, 5.0, 1.0)]
    z = torch.stack(rows).to(TYPES[t])
    targets = torch.arange(len(rows), device="cuda").to(torch.int32) * 7
    for K in (1, 5, 20, 32):
        check_fwd(z, targets, None, K)
    check_fwd(z.repeat(40, 1), targets.repeat(40), None, 9)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [5, 300, 9001])
def test_forward_masked_and_extreme_logits(t, V):
    low = torch.finfo(TYPES[t]).min
    z, targets, _ = make(9, V, t, V)
    z = z.clone()
    z[0] = -math.inf                       # nothing left
    z[1] = -math.inf
    z[1, V // 2] = 1.5                     # one token left
    z[2] = low                             # the type's lowest value everywhere: uniform
    z[3, ::2] = -math.inf
    z[4, 1:] = low
    z[5, 0] = 300.0                        # everything else vanishes
    z[6, : V // 2] = low
    z[7] = -math.inf
    z[7, -2:] = torch.tensor([2.0, 2.0])
    z[8] = 60000.0 if t == "f16" else 1e6  # a large common offset
    targets = torch.tensor([0, V // 2, 1, 1, 0, 0, V - 1, V - 1, 2], dtype=torch.int32, device="cuda")
    check_fwd(z, targets, None, 6)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 0.003, 0.02, 40.0, 3000.0])
def test_forward_and_gradient_over_scales(t, scale):
    z, targets, mask = make(30, 5003, t, 3)
    z = z.clone()
    z[1, ::2] = -math.inf
    z[2, 1:] = torch.finfo(z.dtype).min
    targets[1], targets[2] = 1, 0
    _, _, lse, _, _ = check_fwd(z, targets, mask, 4, scale)
    g = torch.randn(30, device="cuda")
    check_bwd(z, targets, mask, g, g, None, None, scale)


@pytest.mark.parametrize("t,low", [("bf16", -1e4), ("bf16", -1e9), ("f32", -1e9), ("f16", -6e4), ("f32", -1e20), ("f16", -65504.0)])
def test_rows_of_finite_mask_values(t, low):
    z, targets, _ = make(6, 3001, t, 8)
    z = z.clone()
    z[0, 7:] = low                          # a few tokens left
    z[1] = low                              # none left: uniform
    z[2] = low
    z[2, ::2] = -math.inf                   # and some excluded altogether
    z[3, :-1] = low
    targets[:4] = torch.tensor([3, 5, 1, 3000])
    _, _, lse, _, _ = check_fwd(z, targets, None, 4)
    g = torch.randn(6, device="cuda")
    ok = lse.abs() < 2.0 ** 24              # beyond, fp32 log-sum-exps carry no probabilities
    zz, tt, gg = z[ok].contiguous(), targets[ok].contiguous(), g[ok].contiguous()
    check_bwd(zz, tt, None, gg, gg, None, None)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("V", [6, 4096, 30011])
def test_forward_rows_with_nan_or_inf(bad, V):
    z, targets, _ = make(5, V, "bf16", V)
    z = z.clone()
    z[1, V // 3] = bad
    z[3, V - 1] = bad
    if bad == math.inf:
        # +inf leads the order
        _, _, _, _, ids = check_fwd(z, targets, None, 3, status=B_NONFINITE)
        assert int(ids[1, 0]) == V // 3 and int(ids[3, 0]) == V - 1
    else:
        check_fwd(z, targets, None, 3, status=B_NONFINITE)
    # the same rows masked: they are not read
    mask = torch.tensor([1, 0, 1, 0, 1], dtype=torch.uint8, device="cuda")
    check_fwd(z, targets, mask, 3)


B_NONFINITE, B_TARGET = -7, -5


def test_forward_target_outside_the_vocabulary():
    z, targets, _ = make(4, 999, "f32", 0)
    lp, ent = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    targets[2] = 999
    B.oapl_logits_logprobs(B.make_logits(z, targets), lp, ent, None, None, None, st)
    assert int(st) == B_TARGET and bool(torch.isnan(lp[2])) and bool(torch.isfinite(lp[[0, 1, 3]]).all())
    assert bool(torch.isfinite(ent).all())
    # on a masked row it does not matter
    st.zero_()
    mask = torch.tensor([1, 1, 0, 1], dtype=torch.uint8, device="cuda")
    B.oapl_logits_logprobs(B.make_logits(z, targets, mask), lp, None, None, None, None, st)
    assert int(st) == 0 and float(lp[2]) == 0.0


def test_forward_offsets_beyond_32_bits():
    # 17000 rows of 152064 logits: the last rows start past 2^31 elements.  Few rows are live.
    N, V = 17000, 152064
    z = torch.empty(N, V, dtype=torch.bfloat16, device="cuda")
    rows = [0, N // 2, N - 2, N - 1]
    g = torch.Generator(device="cuda").manual_seed(5)
    for r in rows:
        z[r].normal_(0.0, 2.0, generator=g)
    mask = torch.zeros(N, dtype=torch.uint8, device="cuda")
    mask[rows] = 1
    targets = torch.full((N,), 17, dtype=torch.int32, device="cuda")
    lp, ent, lse = (torch.full((N,), 3.0, device="cuda") for _ in range(3))
    ids = torch.zeros(N, 4, dtype=torch.int32, device="cuda")
    L = B.make_logits(z, targets, mask)
    B.oapl_logits_logprobs(L, lp, ent, lse, None, ids)
    r = ref_fwd(z[rows], targets[rows], torch.ones(4, device="cuda"), 4)
    assert torch.equal(ids[rows].long(), r["id"])
    assert float((lp[rows] - r["logp"]).abs().max()) < 1e-4
    dead = mask == 0
    assert float(lp[dead].abs().max()) == 0.0 and bool((ids[dead] == -1).all())
    # and the gradient, in place
    B.oapl_logits_logprobs_bwd(L, lse, ent, torch.ones(N, device="cuda"), None, None, None, z)
    assert float(z[N - 1].float().sum().abs()) < 0.05 and float(z[N - 1, 17]) > 0.9
    assert bool((z[N - 3] == 0).all())


# ---------------------------------------------------------------------------------------- gradient

def ref_bwd(z, targets, mask, lse, ent, gl, ge, gt, ids, scale):
    lp = z.double() * scale - lse.double()[:, None]
    p = torch.where(lse[:, None] < -1e30, 0.0, torch.exp(lp))      # nothing but masked logits in the row
    G = torch.zeros(z.shape[0], dtype=torch.float64, device=z.device)
    point = torch.zeros(z.shape, dtype=torch.float64, device=z.device)
    V = z.shape[1]
    if gl is not None:
        ok = (targets >= 0) & (targets < V)
        G += torch.where(ok, gl.double(), 0.0)
        point.scatter_add_(1, targets.long().clamp(0, V - 1)[:, None], torch.where(ok, gl.double(), 0.0)[:, None])
    if gt is not None:
        ok = (ids >= 0) & (ids < V)
        w = torch.where(ok, gt.double(), 0.0)
        G += w.sum(1)
        point.scatter_add_(1, ids.long().clamp(0, V - 1), w)
    inner = G[:, None].expand(z.shape).clone()
    part = torch.zeros_like(inner)
    if ge is not None:
        part = ge.double()[:, None] * (torch.where(p > 0, lp, torch.zeros_like(lp)) + ent.double()[:, None])
    d = scale * (-torch.where(p > 0, p * (inner + part), torch.zeros_like(p)) + point)
    live = mask.bool()[:, None]
    factor = scale * (inner.abs() + part.abs() * 2 + (ge.double().abs()[:, None] if ge is not None else 0.0))
    dist = (z.double() * scale).abs().nan_to_num(0, 0, 0) + lse.double().abs().nan_to_num(0, 0, 0)[:, None]
    zero = torch.zeros_like(d)
    return tuple(torch.where(live, x, zero) for x in (d, factor * p, dist, point.abs() * scale, factor))


def check_bwd(z, targets, mask, gl, ge, gt, ids, scale=1.0, pad=0, offset=0):
    N, V = z.shape
    lse, ent = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    L = B.make_logits(z, targets, mask, scale)
    B.oapl_logits_logprobs(L, None, ent, lse)
    flat = torch.full((N * (V + pad) + offset,), 5.0, dtype=z.dtype, device="cuda")
    d = flat[offset:].view(N, V + pad)[:, :V]
    B.oapl_logits_logprobs_bwd(L, lse, ent, gl, ge, gt, ids, d)
    m = mask if mask is not None else torch.ones(N, device="cuda")
    want, size, dist, point, factor = ref_bwd(z, targets, m, lse, ent, gl, ge, gt, ids, scale)
    fi = torch.finfo(z.dtype)
    # one rounding to the type; p: 2^-22 of the exponential and three roundings of an exponent of size dist;
    # a few roundings of the factors and of the sum with the point term
    tol = fi.eps / 2 * want.abs() + size * (2.0 ** -22 + (3 * dist + 8 + gt_terms(gt)) * U) * (1 + fi.eps) + (4 + gt_terms(gt)) * U * point
    # p below the smallest normal fp32 number, 2^-126, is 0 there: off by no more than that times its factor
    tol = tol + fi.smallest_normal * fi.eps + 1e-37 + factor * 2.0 ** -126
    close(d, want, tol, "dlogits")
    if pad:
        assert bool((flat[offset:].view(N, V + pad)[:, V:] == 5.0).all())
    assert bool((flat[:offset] == 5.0).all())
    return L, lse, ent, d


def gt_terms(gt):
    return 0 if gt is None else gt.shape[1]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [1, 3, 9, 257, 1000, 8200, 30011])
@pytest.mark.parametrize("offset,pad,doff,dpad", [(0, 0, 0, 0), (3, 5, 3, 5), (1, 2, 4, 0)])
def test_gradient_sizes(t, V, offset, pad, doff, dpad):
    for N, K in [(1, 0), (13, 5), (40, 32)]:
        z, targets, mask = make(N, V, t, V + N, offset, pad)
        g = torch.Generator(device="cuda").manual_seed(N)
        gl, ge = (torch.randn(N, device="cuda", generator=g) for _ in range(2))
        gt = torch.rand(N, K, device="cuda", generator=g) if K else None
        ids = torch.randint(-1, V, (N, K), device="cuda", generator=g).to(torch.int32) if K else None   # repeats, and -1
        check_bwd(z, targets, mask, gl, ge, gt, ids, 1.0, dpad, doff)
        check_bwd(z, targets, None, gl, None, None, None, 1.7, dpad, doff)
        check_bwd(z, targets, None, None, ge, None, None, 0.5, dpad, doff)
        if K:
            check_bwd(z, None if K == 5 else targets, None, None, None, gt, ids, 1.0, dpad, doff)


@pytest.mark.parametrize("t,N,V,pad,dpad", [("bf16", 3700, 5, 0, 3), ("f16", 3700, 2056, 0, 0), ("bf16", 3700, 8200, 3, 3),
                                            ("f32", 1900, 20003, 1, 5), ("bf16", 1800, 40009, 7, 7), ("f16", 901, 131100, 4, 4)])
def test_gradient_many_rows(t, N, V, pad, dpad):
    # a CTA takes several batches of a row; entries with a point term in any of them
    z, targets, mask = make(N, V, t, V, 0, pad)
    g = torch.Generator(device="cuda").manual_seed(N)
    gl, ge = (torch.randn(N, device="cuda", generator=g) for _ in range(2))
    gt = torch.rand(N, 9, device="cuda", generator=g)
    ids = torch.randint(-1, V, (N, 9), device="cuda", generator=g).to(torch.int32)
    L, lse, ent, d = check_bwd(z, targets, mask, gl, ge, gt, ids, 1.0, dpad)
    d = d.clone()
    B.oapl_logits_logprobs_bwd(L, lse, ent, gl, ge, gt, ids, z)        # over the logits
    assert torch.equal(d, z)


def test_gradient_target_among_the_alternatives_and_ids_outside():
    z, targets, _ = make(6, 500, "f32", 2)
    ids = torch.stack([targets, targets, torch.full_like(targets, 500), torch.full_like(targets, -5)], 1).contiguous()
    gt = torch.tensor([[0.5, 0.25, 9.0, 9.0]], device="cuda").repeat(6, 1)
    gl = torch.ones(6, device="cuda")
    targets = targets.clone()
    targets[3] = 501
    check_bwd(z, targets, None, gl, None, gt, ids)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_gradient_masked_logits_and_empty_rows(t):
    z, targets, _ = make(7, 2000, t, 4)
    z = z.clone()
    z[0, ::3] = -math.inf
    z[1] = -math.inf
    z[1, 5] = 0.0
    z[2, 10:] = torch.finfo(z.dtype).min
    z[3] = -math.inf                               # no finite logit
    z[4] = torch.finfo(z.dtype).min if t != "f16" else -math.inf     # nothing but the type's lowest value
    g = torch.randn(7, device="cuda")
    targets[0], targets[3] = 0, 7
    L, lse, ent, d = check_bwd(z, targets, None, g, g, None, None)
    assert int((d[4] != 0).sum()) == 1
    assert bool(torch.isneginf(lse[3])) and float(d[3].double().sum()) == pytest.approx(float(g[3].to(z.dtype)), rel=1e-6)


@pytest.mark.parametrize("t,V", [("bf16", 30011), ("f16", 50024), ("f32", 4097)])
def test_gradient_in_place_and_repeatable(t, V):
    z, targets, mask = make(57, V, t, 9)
    g = torch.randn(57, device="cuda")
    gt, ids = torch.rand(57, 6, device="cuda"), torch.randint(0, V, (57, 6), device="cuda").to(torch.int32)
    L, lse, ent, d = check_bwd(z, targets, mask, g, g, gt, ids)
    again = torch.empty_like(d)
    B.oapl_logits_logprobs_bwd(L, lse, ent, g, g, gt, ids, again)
    assert torch.equal(d, again)
    B.oapl_logits_logprobs_bwd(L, lse, ent, g, g, gt, ids, z)
    assert torch.equal(d, z)


def test_gradient_against_differences_and_autograd():
    N, V, K = 3, 23, 4
    g = torch.Generator().manual_seed(0)
    z = torch.randn(N, V, generator=g).double()
    w_lp, w_h, w_t = torch.randn(N, generator=g).double(), torch.randn(N, generator=g).double(), torch.randn(N, K, generator=g).double()
    targets = torch.tensor([0, 22, 7])
    ids = torch.tensor([[1, 2, 3, 4], [22, 0, 5, 6], [9, 9, 7, 1]])
    scale = 1.3

    def value(x):
        lp = torch.log_softmax(scale * x, 1)
        return ((w_lp * lp.gather(1, targets[:, None])[:, 0]).sum() - (w_h * (lp.exp() * lp).sum(1)).sum()
                + (w_t * lp.gather(1, ids)).sum())
    x = z.clone().requires_grad_()
    value(x).backward()
    h = 1e-5
    for n, v in [(0, 0), (1, 22), (2, 9), (2, 7), (1, 11)]:
        e = torch.zeros_like(z)
        e[n, v] = h
        assert float((value(z + e) - value(z - e)) / (2 * h)) == pytest.approx(float(x.grad[n, v]), abs=1e-8)
    zc = z.float().cuda()
    L = B.make_logits(zc, targets.to(torch.int32).cuda(), None, scale)
    lse, ent, d = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(zc)
    B.oapl_logits_logprobs(L, None, ent, lse)
    B.oapl_logits_logprobs_bwd(L, lse, ent, w_lp.float().cuda(), w_h.float().cuda(), w_t.float().cuda(),
                               ids.to(torch.int32).cuda(), d)
    # every entry is a sum of a few terms of size <= 4, each with a few roundings of 2^-24
    assert float((d.cpu().double() - x.grad).abs().max()) <= 4 * 20 * U + 2.0 ** -21


# ---------------------------------------------------------------------------------------- streams, graphs

def test_other_stream_and_two_calls_at_once():
    a, b = make(64, 50021, "bf16", 1), make(64, 50021, "f32", 2)
    want = [check_fwd(*x, 8) for x in (a, b)]
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for (z, t, m), s in zip((a, b), streams):
        with torch.cuda.stream(s):
            o = [torch.empty(64, device="cuda") for _ in range(3)] + [torch.empty(64, 8, device="cuda"),
                                                                        torch.empty(64, 8, dtype=torch.int32, device="cuda")]
            for _ in range(20):
                B.oapl_logits_logprobs(B.make_logits(z, t, m), *o)
            outs.append(o)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(o, w))


def test_captured_and_replayed():
    z, targets, mask = make(33, 30011, "bf16", 6)
    o = [torch.zeros(33, device="cuda") for _ in range(3)]
    d, g = torch.zeros_like(z), torch.randn(33, device="cuda")
    L = B.make_logits(z, targets, mask)

    def step():
        B.oapl_logits_logprobs(L, *o)
        B.oapl_logits_logprobs_bwd(L, o[2], o[1], g, g, None, None, d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    z2, _, _ = make(33, 30011, "bf16", 7)
    z.copy_(z2)
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in o] + [d.clone()]
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, o + [d]))


def test_single_outputs():
    z, targets, _ = make(9, 3001, "bf16", 5)
    lp, ent, lse, top, ids = check_fwd(z, targets, None, 6)
    L, new = B.make_logits(z, targets), lambda x: torch.full_like(x, 3)
    for k, want in enumerate((lp, ent, lse, top, ids)):
        args = [None] * 5
        args[k] = new(want)
        B.oapl_logits_logprobs(L, *args)
        assert torch.equal(args[k], want)
    one = new(ent)
    B.oapl_logits_logprobs(B.make_logits(z), None, one)         # no targets needed for the entropy
    assert torch.equal(one, ent)


def test_binding_refuses_tensors_of_another_device():
    with pytest.raises(ValueError):
        B._stream_of(torch.cuda.current_device() + 1)


def test_binding_refusals():
    z, targets, mask = make(4, 64, "bf16", 0)
    f = torch.empty(4, device="cuda")
    L = B.make_logits(z, targets, mask)
    with pytest.raises(TypeError):
        B.make_logits(z.t())
    with pytest.raises(TypeError):
        B.make_logits(z, targets.long())
    with pytest.raises(TypeError):
        B.make_logits(z, targets, mask[:3])
    with pytest.raises(TypeError):
        B.oapl_logits_logprobs(L, f[:3])
    with pytest.raises(TypeError):
        B.oapl_logits_logprobs(L, f.double())
    with pytest.raises(B.OaplError) as e:
        B.oapl_logits_logprobs(L, f, top_id=torch.empty(4, 33, dtype=torch.int32, device="cuda"))
    assert e.value.status == -1
    with pytest.raises(B.OaplError):
        B.oapl_logits_logprobs(B.make_logits(z), f)          # no targets
    with pytest.raises(TypeError):
        B.oapl_logits_logprobs_bwd(L, f, f, f, None, None, None, z.float())
