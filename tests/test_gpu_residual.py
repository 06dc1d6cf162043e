"""oapl_residual_norm and its gradient against plain 64-bit forms of the same definitions."""
import itertools

import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24
SUM = 60 * U    # a sum over a row: at most 32 terms a thread, 9 levels of tree, the terms' own roundings


def half_step(want, t):
    f = torch.finfo(t)
    return want.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def rand(g, N, d, t, pad=0, offset=0, std=1.0):
    flat = torch.randn(N * (d + pad) + offset, device="cuda", generator=g).mul_(std).to(TYPES[t])
    return flat[offset:].view(N, d + pad)[:, :d]


def make(N, d, t, gate="none", post=True, pre=True, weight=None, pad=0, offset=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + d)
    weight = weight or t
    c = dict(t=t, eps=1e-5, a=0.75, b=1.25, off=0.5 if post else 0.0)
    c["x"], c["y"] = rand(g, N, d, t, pad, offset, 2.0), rand(g, N, d, t, pad, offset, 0.5)
    if d > 8:
        c["x"][:, 3] *= 30
    c["gate"] = {"none": lambda: None, "row": lambda: rand(g, N, 1, "f32"), "column": lambda: rand(g, 1, d, weight)[0],
                 "full": lambda: rand(g, N, d, t, pad, offset)}[gate]()
    c["kind"] = gate
    c["w_post"] = rand(g, 1, d, weight)[0] if post else None
    c["w_pre"] = rand(g, 1, d, weight)[0] if pre else None
    c["dh"] = rand(g, N, d, t, pad, offset) if pre else None
    c["dxo"] = rand(g, N, d, t, pad, offset)
    return c


def wide(t):
    return None if t is None else t.double()


def like(x, pad=16):
    """A matrix of x's shape and type with guarded columns behind it, which keep 16-byte rows where d has them."""
    N, d = x.shape
    whole = torch.full((N, d + pad), 7.0, dtype=x.dtype, device="cuda")
    return whole, whole[:, :d]


def struct(c):
    return B.make_residual(c["x"], c["y"], c["gate"], c["w_post"], c["w_pre"], c["eps"], c["a"], c["b"], c["off"])


def scalars(c):
    f = lambda v: torch.tensor(v, dtype=torch.float32).item()  # noqa: E731
    return f(c["eps"]), f(c["a"]), f(c["b"]), f(c["off"])


def ref_fwd(c):
    eps, a, b, off = scalars(c)
    x, y = wide(c["x"]), wide(c["y"])
    r = {}
    u = 0.0
    if y is not None:
        u = y
        if c["w_post"] is not None:
            r["rp"] = (y.square().mean(1) + eps).rsqrt()
            u = y * r["rp"][:, None] * (wide(c["w_post"]) + off)
        if c["gate"] is not None:
            u = u * wide(c["gate"])
        u = u * b
    r["xo"] = a * x + u
    size = (a * x).abs() + (u.abs() if y is not None else 0.0)
    r["t_xo"] = SUM * size
    if c["w_pre"] is not None:
        r["rq"] = (r["xo"].square().mean(1) + eps).rsqrt()
        # a relative error of the mean square: its own roundings, and those of x' (cancelled terms count in full)
        spoiled = SUM * (size.square().mean(1).sqrt() * r["rq"])[:, None]
        w = (wide(c["w_pre"]) + off)
        r["h"] = r["xo"] * r["rq"][:, None] * w
        r["t_h"] = (w * r["rq"][:, None]).abs() * r["t_xo"] + r["h"].abs() * (SUM + spoiled)
        r["t_rq"] = r["rq"] * (SUM + spoiled[:, 0])
    return r


def within(got, want, tol, what):
    off = (got.double() - want).abs()
    assert bool((off <= tol + half_step(want, got.dtype)).all()), (what, float((off - tol - half_step(want, got.dtype)).max()))


def check_fwd(c):
    N, d = c["x"].shape
    (gx, xo), (gh, h) = like(c["x"]), like(c["x"])
    rp = torch.empty(N, device="cuda") if c["w_post"] is not None else None
    rq = torch.empty(N, device="cuda") if c["w_pre"] is not None else None
    B.oapl_residual_norm(struct(c), xo, h if rq is not None else None, rp, rq)
    r = ref_fwd(c)
    within(xo, r["xo"], r["t_xo"], "x_out")
    assert bool((gx[:, d:] == 7).all()) and bool((gh[:, d:] == 7).all())
    if rp is not None:
        within(rp, r["rp"], SUM * r["rp"], "rstd_post")
    if rq is not None:
        within(h, r["h"], r["t_h"], "h")
        within(rq, r["rq"], r["t_rq"], "rstd_pre")
    return xo, h, rp, rq


def ref_bwd(c, xo, rp, rq):
    """The gradient by its formulas, with a bound of the kernel's rounding beside each value."""
    eps, a, b, off = scalars(c)
    d = c["dxo"].shape[1]
    t = wide(c["dxo"])
    tol = 4 * U * t.abs()
    r = {}
    m1r = torch.zeros(t.shape[0], 1, dtype=torch.float64, device="cuda")
    if c["w_pre"] is not None:
        rr = rq.double()[:, None]
        xh, dh = wide(xo) * rr, wide(c["dh"])
        q = dh * (wide(c["w_pre"]) + off)
        m1, m1_abs = (q * xh).mean(1, keepdim=True), (q * xh).abs().mean(1, keepdim=True)
        t = t + rr * (q - xh * m1)
        tol = tol + 6 * U * rr * (q.abs() + (xh * m1).abs()) + rr * xh.abs() * SUM * m1_abs
        r["dw_pre"], s = (dh * xh).sum(0), (dh * xh).abs().sum(0)
        r["t_dw_pre"] = (t.shape[0] + 16) * U * s
        m1r, m1e = rr * m1.abs(), rr * SUM * m1_abs
    r["dx"], r["t_dx"] = a * t, abs(a) * tol
    if c["y"] is None:
        return r
    yh = wide(c["y"]) * (rp.double()[:, None] if rp is not None else 1.0)
    w = wide(c["w_post"]) + off if rp is not None else torch.ones(d, dtype=torch.float64, device="cuda")
    u = yh * w
    g = wide(c["gate"]) if c["gate"] is not None else 1.0
    gate = b * t * u
    t_gate = (b * u).abs() * tol + 6 * U * gate.abs()
    e = b * g * t
    t_e = (b * g * torch.ones_like(t)).abs() * tol + 4 * U * e.abs()
    # the row's mean of A t, A = b u (without a row's gate), formed from two sums
    A = (b * u * (g if c["kind"] in ("column", "full") else 1.0)).abs()
    parts = wide(c["dxo"]).abs() + (rr * q.abs() if c["w_pre"] is not None else 0.0)
    t_mean = SUM * (A * parts).mean(1, keepdim=True) + (A * tol).mean(1, keepdim=True)
    if c["w_pre"] is not None:
        t_mean = t_mean + (SUM * m1r + m1e) * (A * xh.abs()).mean(1, keepdim=True)
    if c["kind"] == "row":
        r["dg"], r["t_dg"] = gate.sum(1, keepdim=True), t_mean * d
    elif c["kind"] == "column":
        r["dg"], r["t_dg"] = gate.sum(0), t_gate.sum(0) + (t.shape[0] + 16) * U * gate.abs().sum(0)
    elif c["kind"] == "full":
        r["dg"], r["t_dg"] = gate, t_gate
    if rp is not None:
        r["dw_post"] = (e * yh).sum(0)
        r["t_dw_post"] = (t_e * yh.abs()).sum(0) + (t.shape[0] + 16) * U * (e * yh).abs().sum(0)
        rr = rp.double()[:, None]
        m2 = (w * e * yh).mean(1, keepdim=True)
        t_m2 = t_mean * (g.abs() if c["kind"] == "row" else 1.0) + 4 * U * m2.abs()
        r["dy"] = rr * (w * e - yh * m2)
        r["t_dy"] = rr * (w.abs() * t_e + yh.abs() * t_m2 + 6 * U * ((w * e).abs() + (yh * m2).abs()))
    else:
        r["dy"], r["t_dy"] = e, t_e
    return r


def workspace(N, d):
    return torch.full((B.oapl_residual_norm_workspace_bytes(N, d),), 0xFF, dtype=torch.uint8, device="cuda")


def check_bwd(c, accumulate=False):
    N, d = c["x"].shape
    # x' and the statistics as a forward pass leaves them
    r = ref_fwd(c)
    xo = like(c["x"], c["x"].stride(0) - d if N > 1 else 0)[1]
    xo.copy_(r["xo"])
    rp, rq = (r[k].float() if k in r else None for k in ("rp", "rq"))
    (gx, dx), (gy, dy) = like(c["x"]), like(c["x"])
    new = lambda *s: torch.full(s, 3.0 if accumulate else float("nan"), device="cuda")  # noqa: E731
    has_y = c["y"] is not None
    dg = {"none": lambda: None, "row": lambda: new(N, 1), "column": lambda: new(d), "full": lambda: like(c["x"])[1]}[c["kind"]]()
    dwp, dwq = new(d) if rp is not None else None, new(d) if rq is not None else None
    B.oapl_residual_norm_bwd(struct(c), xo if rq is not None else None, rp, rq, c["dh"], c["dxo"], dx, dy if has_y else None, dg,
                             dwp, dwq, accumulate, workspace(N, d))
    w = ref_bwd(c, xo, rp, rq)
    within(dx, w["dx"], w["t_dx"], "dx")
    assert bool((gx[:, d:] == 7).all()) and bool((gy[:, d:] == 7).all())
    add = 3.0 if accumulate else 0.0
    if has_y:
        within(dy, w["dy"], w["t_dy"], "dy")
        if dg is not None:
            within(dg, w["dg"] + (add if c["kind"] == "column" else 0.0), w["t_dg"], "dgate")
    if dwp is not None:
        within(dwp, w["dw_post"] + add, w["t_dw_post"], "dw_post")
    if dwq is not None:
        within(dwq, w["dw_pre"] + add, w["t_dw_pre"], "dw_pre")


KINDS = ["none", "row", "column", "full"]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("d", [1, 2, 7, 8, 33, 64, 257, 512, 520, 1111, 2048, 2056, 3584, 4097, 8192])
@pytest.mark.parametrize("gate", KINDS)
def test_sizes_and_gates(t, d, gate):
    for N, pad, offset in [(1, 0, 0), (3, 8, 0), (70, 1, 1)]:
        c = make(N, d, t, gate, pad=pad, offset=offset)
        check_fwd(c)
        check_bwd(c, accumulate=N == 3)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("d", [9001, 12288, 16383, 16384])
def test_widest_rows(t, d):
    for N in (2, 300):
        c = make(N, d, t, "full")
        check_fwd(c)
        check_bwd(c)


@pytest.mark.parametrize("t,weight", [("bf16", "f32"), ("f16", "bf16"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "f16")])
@pytest.mark.parametrize("d", [64, 1000, 1001])
def test_weights_of_another_type(t, weight, d):
    for gate in ("none", "column"):
        c = make(40, d, t, gate, weight=weight)
        check_fwd(c)
        check_bwd(c)


@pytest.mark.parametrize("post,pre", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("gate", KINDS)
@pytest.mark.parametrize("d", [72, 1536, 3001])
def test_parts_left_out(post, pre, gate, d):
    c = make(90, d, "bf16", gate, post, pre)
    check_fwd(c)
    check_bwd(c)


def test_the_norm_alone():
    for t, d in itertools.product(TYPES, (64, 1001, 3584)):
        c = make(50, d, t)
        c.update(y=None, w_post=None)
        check_fwd(c)
        check_bwd(c)


@pytest.mark.parametrize("t,N,d,gate", [("bf16", 3000, 3584, "column"), ("bf16", 5000, 256, "row"), ("f32", 2001, 1111, "full"),
                                        ("f16", 40000, 64, "column"), ("bf16", 1200, 5120, "none"), ("f32", 1300, 4096, "column"),
                                        ("bf16", 2000, 3001, "column"), ("bf16", 30000, 77, "row"), ("f32", 9000, 201, "full"),
                                        ("f16", 4000, 511, "column"), ("f16", 1000, 8191, "none"), ("f32", 700, 7313, "full"),
                                        ("f32", 500, 7600, "full"), ("bf16", 300, 12001, "column")])
def test_many_rows(t, N, d, gate):
    c = make(N, d, t, gate)
    check_fwd(c)
    check_bwd(c)


def test_rows_of_zeros_and_what_is_not_finite_stay_in_their_rows():
    for d in (256, 1536, 1537):
        c = make(40, d, "bf16")
        c["off"] = 0.0
        for k in ("x", "y", "dh", "dxo"):
            c[k][5] = 0
        c["y"][9, 2], c["x"][11, 7] = float("inf"), float("nan")
        xo, h = torch.empty_like(c["x"]), torch.empty_like(c["x"])
        rp, rq = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
        B.oapl_residual_norm(struct(c), xo, h, rp, rq)
        assert bool((xo[5] == 0).all()) and bool((h[5] == 0).all())
        good = torch.tensor([i not in (9, 11) for i in range(40)], device="cuda")
        assert bool(torch.isfinite(h[good]).all()) and not bool(torch.isfinite(h[9]).all()) and bool(torch.isnan(h[11]).all())
        dx, dy = torch.empty_like(c["x"]), torch.empty_like(c["x"])
        B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], c["dxo"], dx, dy)
        assert bool((dx[5] == 0).all()) and bool((dy[5] == 0).all()) and bool(torch.isfinite(dx[good]).all())


@pytest.mark.parametrize("d", [256, 1536, 1537])
@pytest.mark.parametrize("gate", ["column", "full"])
def test_results_over_inputs(d, gate):
    N = 500
    c = make(N, d, "bf16", gate)
    want = [t.clone() for t in check_fwd(c)]
    for keys in (("x", "y"), ("y", "x")) + ((("gate", "x"), ("x", "gate")) if gate == "full" else ()):
        e = dict(c, **{k: c[k].clone() for k in keys})
        rp, rq = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        B.oapl_residual_norm(struct(e), e[keys[0]], e[keys[1]], rp, rq)
        assert torch.equal(e[keys[0]], want[0]) and torch.equal(e[keys[1]], want[1]) and torch.equal(rq, want[3])
    xo, _, rp, rq = want
    dx, dy = torch.empty_like(xo), torch.empty_like(xo)
    dg = torch.empty_like(xo) if gate == "full" else None
    B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], c["dxo"], dx, dy, dg)
    places = ["xo", "dh", "dxo", "y"] + (["gate"] if gate == "full" else [])
    for p, q in itertools.permutations(places, 2):
        e = dict(c, xo=xo)
        e = {**e, **{k: e[k].clone() for k in places}}
        dg2 = torch.empty_like(xo) if gate == "full" else None
        B.oapl_residual_norm_bwd(struct(e), e["xo"], rp, rq, e["dh"], e["dxo"], e[p], e[q], dg2)
        assert torch.equal(e[p], dx) and torch.equal(e[q], dy), (p, q)
        assert dg is None or torch.equal(dg, dg2)


def test_gradient_without_some_results_is_the_same():
    N, d = 300, 640
    c = make(N, d, "bf16", "column")
    xo, _, rp, rq = check_fwd(c)
    names = ("dx", "dy", "dgate", "dw_post", "dw_pre")
    new = lambda: dict(dx=torch.empty(N, d, dtype=torch.bfloat16, device="cuda"), dy=torch.empty(N, d, dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                       dgate=torch.empty(d, device="cuda"), dw_post=torch.empty(d, device="cuda"), dw_pre=torch.empty(d, device="cuda"))
    want = new()
    B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], c["dxo"], **want, ws=workspace(N, d))
    for k in names:
        got = new()
        B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], c["dxo"], **{k: got[k]}, ws=workspace(N, d))
        assert torch.equal(got[k], want[k]), k
    # no gradient of x' from elsewhere: as zeros
    got, zero = new(), new()
    B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], None, **got, ws=workspace(N, d))
    B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], torch.zeros_like(c["dxo"]), **zero, ws=workspace(N, d))
    assert all(torch.equal(got[k], zero[k]) for k in names)


def test_forward_without_results_that_are_not_asked_for():
    c = make(33, 1024, "bf16", "row")
    xo, h, rp, rq = check_fwd(c)
    h2, xo2 = torch.empty_like(c["x"]), torch.empty_like(c["x"])
    B.oapl_residual_norm(struct(c), None, h2)
    assert torch.equal(h, h2)
    B.oapl_residual_norm(struct(c), xo2, h2, None, None)
    assert torch.equal(xo, xo2)


@pytest.mark.parametrize("gate", KINDS)
def test_gradient_against_autograd_and_differences(gate):
    N, d = 24, 48
    c = make(N, d, "f32", gate)
    eps, a, b, off = scalars(c)
    leaves = {k: c[k].double().requires_grad_() for k in ("x", "y", "w_post", "w_pre") + (("gate",) if gate != "none" else ())}

    def loss(v):
        n = lambda m: m / (m.square().mean(1, keepdim=True) + eps).sqrt()  # noqa: E731
        u = n(v["y"]) * (v["w_post"] + off)
        xo = a * v["x"] + b * (u * v["gate"] if gate != "none" else u)
        return (n(xo) * (v["w_pre"] + off) * c["dh"].double()).sum() + (xo * c["dxo"].double()).sum()

    want = dict(zip(leaves, torch.autograd.grad(loss(leaves), list(leaves.values()))))
    xo, h = torch.empty_like(c["x"]), torch.empty_like(c["x"])
    rp, rq = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    B.oapl_residual_norm(struct(c), xo, h, rp, rq)
    got = dict(x=torch.empty(N, d, device="cuda"), y=torch.empty(N, d, device="cuda"), w_post=torch.empty(d, device="cuda"),
               w_pre=torch.empty(d, device="cuda"))
    if gate != "none":
        got["gate"] = torch.empty_like(c["gate"])
    B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], c["dxo"], got["x"], got["y"], got.get("gate"), got["w_post"], got["w_pre"],
                             ws=workspace(N, d))
    for k in want:
        # fp32 throughout: a few hundred half steps of the largest term
        assert float((got[k].double() - want[k]).abs().max()) <= 300 * U * float(want[k].abs().max() + 1), k
        # central differences of the 64-bit loss along a random direction
        e = torch.randn_like(want[k])
        h_ = 1e-4
        up, down = ({**{j: v.detach() for j, v in leaves.items()}, k: leaves[k].detach() + s * h_ * e} for s in (1, -1))
        slope = float((loss(up) - loss(down)) / (2 * h_))
        along = float((got[k].double() * e).sum())
        assert abs(slope - along) <= 1e-4 * float((want[k] * e).abs().sum()) + 1e-6, k


def test_repeats_bit_for_bit_on_another_stream_and_captured():
    N, d = 2000, 1536
    c = make(N, d, "bf16", "column")
    xo, _, rp, rq = check_fwd(c)
    ws = workspace(N, d)
    new = lambda: [torch.empty(N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [torch.empty(d, device="cuda") for _ in range(3)]  # noqa: E731
    call = lambda o: B.oapl_residual_norm_bwd(struct(c), xo, rp, rq, c["dh"], c["dxo"], *o, False, ws)  # noqa: E731
    want, got = new(), new()
    call(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    x2, h2 = torch.empty_like(c["x"]), torch.empty_like(c["x"])
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            B.oapl_residual_norm(struct(c), x2, h2)
            call(got)
        for _ in range(3):
            for o in got + [x2]:
                o.fill_(float("nan"))
            graph.replay()
    side.synchronize()
    assert torch.equal(x2, xo) and all(torch.equal(a, b) for a, b in zip(want, got))


def test_row_offsets_beyond_32_bits():
    N, d = 280000, 8192        # 2.3e9 elements
    x = torch.empty(N, d, dtype=torch.bfloat16, device="cuda").fill_(1.0)
    x[-1] = torch.linspace(-2, 2, d, device="cuda").bfloat16()
    x[0] = x[-1]
    x[2 ** 31 // d] = x[-1]
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    r = B.make_residual(x, w_pre=w)
    rq = torch.empty(N, device="cuda")
    h = torch.empty_like(x)
    B.oapl_residual_norm(r, None, h, None, rq)
    assert torch.equal(h[-1], h[0]) and torch.equal(h[2 ** 31 // d], h[0])
    want = (x[0].double() * (x[0].double().square().mean() + 1e-6).rsqrt())
    within(h[0], want, SUM * want.abs(), "h")
    assert bool((h[1] == 1).all()) and bool((h[-2] == 1).all())
    B.oapl_residual_norm_bwd(r, x, None, rq, h, None, h)
    assert torch.equal(h[-1], h[0])


def test_binding_refusals():
    x, w = torch.zeros(4, 16, device="cuda"), torch.ones(16, device="cuda")
    r = B.make_residual(x, w_pre=w)
    for bad in (lambda: B.make_residual(x, x.half()), lambda: B.make_residual(x, x[:3]), lambda: B.make_residual(x.t()),
                lambda: B.make_residual(x, x, gate=torch.ones(15, device="cuda")), lambda: B.make_residual(x, x, gate=x.half()),
                lambda: B.make_residual(x, w_pre=w[:8]), lambda: B.make_residual(x, x, w_post=w.half(), w_pre=w),
                lambda: B.oapl_residual_norm(r, x.half(), x), lambda: B.oapl_residual_norm(r, x[:3], x),
                lambda: B.oapl_residual_norm(r, x.clone(), x, rstd_pre=torch.zeros(3, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_residual_norm(r, x.clone(), None)
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_residual_norm(r, x, x)
    with pytest.raises(B.OaplError, match="WORKSPACE_TOO_SMALL"):
        B.oapl_residual_norm_bwd(r, x, None, torch.ones(4, device="cuda"), x.clone(), None, x.clone(), dw_pre=w.clone(),
                                 ws=torch.zeros(64, dtype=torch.uint8, device="cuda"))
