"""oapl_logits_adjust and its gradient against a plain form in 64 bits, row by row."""
import math

import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24


def half_step(want, t):
    f = torch.finfo(t)
    return want.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def pack(allowed):
    """Truth values [rows, V] as words of 32 bits."""
    rows, V = allowed.shape
    b = torch.nn.functional.pad(allowed, (0, (-V) % 32)).view(rows, -1, 32).long()
    w = (b << torch.arange(32, device=b.device)).sum(2)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def make(N, V, t, seed=0, prompt=20, answer=30, bias=5, allowed=0.7, pad=0, offset=0, low=0):
    """Inputs on the GPU, and the rows' histories as lists on the host."""
    g = torch.Generator().manual_seed(seed + V)
    flat = torch.randn(N * (V + pad) + offset, generator=g).mul_(3.0).to(TYPES[t]).cuda()
    c = dict(z=flat[offset:].view(N, V + pad)[:, :V], t=t)
    if prompt or answer:
        # some tokens are outside the vocabulary, some occur many times
        toks = torch.randint(-2, V + 2, (4 * (prompt + answer) + 8,), generator=g)
        toks[::3] = toks[::3] % max(1, min(V, 7))
        s0 = torch.randint(0, toks.numel() - prompt - answer, (N,), generator=g)
        s1 = s0 + torch.randint(0, prompt + 1, (N,), generator=g)
        s2 = s1 + torch.randint(0, answer + 1, (N,), generator=g)
        c.update(tokens=toks.to(torch.int32).cuda(), spans=torch.stack([s0, s1, s2], 1).cuda(),
                 repetition=(torch.rand(N, generator=g) * 1.5 + 0.5).cuda(), frequency=(torch.randn(N, generator=g)).cuda(),
                 presence=torch.randn(N, generator=g).cuda())
    if bias:
        n = torch.randint(0, bias + 1, (N,), generator=g)
        start = torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)])
        total = int(start[-1])
        ids = torch.randint(-1, V + 1, (total,), generator=g)
        ids[::2] = ids[::2] % max(1, min(V, 3))       # the same token several times
        c.update(bias_start=start.cuda(), bias_id=ids.to(torch.int32).cuda(), bias=(4 * torch.randn(total, generator=g)).cuda())
    if allowed is not None:
        c["open"] = torch.rand(N, V, generator=g).cuda() < allowed
        if N > 2:
            c["open"][1] = False          # nothing is allowed
            c["open"][2] = True
        c["allowed"] = pack(c["open"])
    return c


KEYS = ("tokens", "spans", "repetition", "frequency", "presence", "bias_start", "bias_id", "bias", "allowed", "allowed_row")


def args(L, c):
    return B.make_adjust(L, **{k: c.get(k) for k in KEYS})


def parts(c):
    """Per row: counts, seen, slope, biases' sum and magnitude, what is allowed."""
    N, V = c["z"].shape
    one = torch.ones(N, V, dtype=torch.float64)
    count, seen, bias, size = torch.zeros(N, V, dtype=torch.float64), torch.zeros(N, V, dtype=torch.bool), 0 * one, 0 * one
    if c.get("spans") is not None:
        toks, spans = c["tokens"].cpu().long(), c["spans"].cpu().tolist()
        for n, (s0, s1, s2) in enumerate(spans):
            a, p = toks[s1:s2], toks[s0:s1]
            a, p = a[(a >= 0) & (a < V)], p[(p >= 0) & (p < V)]
            count[n] = torch.bincount(a, minlength=V).double()
            seen[n] = (count[n] > 0) | (torch.bincount(p, minlength=V) > 0)
    if c.get("bias_start") is not None:
        start, ids, b = c["bias_start"].cpu().tolist(), c["bias_id"].cpu().tolist(), c["bias"].cpu().double().tolist()
        for n in range(N):
            for i in range(start[n], start[n + 1]):
                if 0 <= ids[i] < V:
                    bias[n, ids[i]] += b[i]
                    size[n, ids[i]] += abs(b[i])
    open_ = c["open"] if c.get("open") is not None else torch.ones(N, V, dtype=torch.bool, device="cuda")
    return count.cuda(), seen.cuda(), bias.cuda(), size.cuda(), open_


def row(c, k, default):
    v = c.get(k)
    return default if v is None else v.double()[:, None]


def check_fwd(c, mask=None, over=False, status=0):
    N, V = c["z"].shape
    z = c["z"].double()
    count, seen, bias, size, open_ = parts(c)
    r, f, p = row(c, "repetition", 1.0), row(c, "frequency", 0.0), row(c, "presence", 0.0)
    z1 = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
    want = z1 - f * count - p * (count > 0) + bias
    touched = seen | (size > 0)
    # four roundings of sums of these terms in fp32, and one for each further bias
    tol = (4 + (size > 0) * 8) * U * (z1.abs() + (f * count).abs() + (p * (count > 0)).abs() + size) * touched
    whole = torch.full((N, V + 16), 7.0, dtype=c["z"].dtype, device="cuda")
    out = c["z"] if over else whole[:, :V]
    before = c["z"].clone()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    L = B.make_logits(c["z"], None, mask)
    B.oapl_logits_adjust(L, args(L, c), out, st)
    live = torch.ones(N, 1, dtype=torch.bool, device="cuda") if mask is None else mask.bool()[:, None]
    bad = open_ & live & ~((out.double() == want) | ((out.double() - want).abs() <= tol + half_step(want, out.dtype)))
    assert not bool(bad.any()), (out[bad][:5], want[bad][:5], bad.nonzero()[:5])
    assert bool((out[(~open_) & live] == -math.inf).all())
    same = open_ & live & ~touched
    assert torch.equal(out[same], before[same])
    gone = ~live.expand_as(open_)
    assert torch.equal(out[gone], before[gone] if over else torch.full_like(out[gone], 7.0))
    assert bool((whole[:, V:] == 7).all()) and int(st) == status
    return out


def check_bwd(c, mask=None, where="apart", status=0):
    N, V = c["z"].shape
    g = torch.Generator(device="cuda").manual_seed(1)
    d = torch.randn(N, V + 16, device="cuda", generator=g).to(c["z"].dtype)[:, :V]
    _, seen, _, _, open_ = parts(c)
    r = row(c, "repetition", 1.0)
    want = d.double() * torch.where(seen, torch.where(c["z"].double() > 0, 1 / r, r * torch.ones_like(d, dtype=torch.float64)), 1.0)
    keep = open_ if mask is None else open_ & mask.bool()[:, None]
    want = torch.where(keep, want, 0.0)
    L = B.make_logits(c["z"], None, mask)
    A = args(L, c)
    whole = torch.full((N, V + 16), 7.0, dtype=d.dtype, device="cuda")
    out = dict(apart=whole[:, :V], d=d, z=c["z"])[where]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_logits_adjust_bwd(L, A, d, out, st)
    assert bool(((out.double() - want).abs() <= half_step(want, out.dtype) + 2 * U * want.abs()).all())
    assert bool((whole[:, V:] == 7).all()) and int(st) == status


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 255, 1000, 2049, 4096, 8200, 20011])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (1, 1)])
def test_sizes(t, V, pad, offset):
    for N in (1, 7):
        c = make(N, V, t, N, pad=pad, offset=offset)
        check_fwd(c)
        check_bwd(c)
        mask = torch.tensor([i % 3 != 1 for i in range(N)], dtype=torch.uint8, device="cuda")
        check_bwd(c, mask)
        check_fwd(c, mask, over=True)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,pad", [(1, 152064, 0), (40, 152064, 0), (90, 50021, 0), (64, 50021, 3), (600, 8192, 0)])
def test_many_rows_and_long_histories(t, N, V, pad):
    c = make(N, V, t, 3, prompt=3000, answer=2500, bias=60, pad=pad)
    check_fwd(c)
    check_bwd(c)
    check_fwd(c, over=True)


@pytest.mark.parametrize("drop", ["repetition", "frequency", "presence", "history", "bias", "allowed", "all"])
@pytest.mark.parametrize("V", [1000, 5001])
def test_parts_left_out(drop, V):
    for over in (False, True):
        c = make(9, V, "bf16", 4)
        gone = dict(history=("tokens", "spans", "repetition", "frequency", "presence"), bias=("bias_start", "bias_id", "bias"),
                    allowed=("allowed", "open"), all=KEYS + ("open",)).get(drop, (drop,))
        for k in gone:
            c.pop(k, None)
        if not over:
            check_bwd(c)
        check_fwd(c, over=over)


def test_histories_of_length_zero_and_one_and_shared_tokens():
    c = make(6, 100, "f32", 5, bias=0, allowed=None)
    c["tokens"] = torch.tensor([5, 5, 7, 99, 0, 5], dtype=torch.int32, device="cuda")
    c["spans"] = torch.tensor([[0, 0, 0], [6, 6, 6], [0, 1, 1], [0, 0, 1], [0, 6, 6], [0, 2, 6]], device="cuda")
    check_fwd(c)
    check_bwd(c)
    c.update(tokens=c["tokens"][:0], spans=torch.zeros(6, 3, dtype=torch.long, device="cuda"))
    check_fwd(c)


@pytest.mark.parametrize("over", [False, True])
@pytest.mark.parametrize("N,V", [(2, 20000), (700, 8300)])
def test_answers_too_long_to_count_in_16_bits(N, V, over):
    # 66000 times one token, 65535 and 65536 tokens beside it
    g = torch.Generator().manual_seed(17)
    toks = torch.cat([torch.full((66000,), 5), torch.randint(0, V, (9000,), generator=g), torch.full((4,), V - 1)])
    c = make(N, V, "f32", 17, prompt=0, answer=0)
    c["tokens"] = toks.to(torch.int32).cuda()
    ends = torch.tensor([toks.numel(), 65535, 65536, 66001, 100, 70000])
    spans = torch.zeros(N, 3, dtype=torch.long)
    spans[:, 2] = ends[torch.arange(N) % 6]
    spans[3::6, 1] = 3
    c.update(spans=spans.cuda(), repetition=torch.full((N,), 1.25, device="cuda"), frequency=torch.full((N,), 0.001, device="cuda"),
             presence=torch.full((N,), -0.5, device="cuda"))
    if not over:
        check_bwd(c)
    check_fwd(c, over=over)


def test_empty_bias_list():
    c = make(4, 300, "bf16", 6, bias=0)
    c.update(bias_start=torch.zeros(5, dtype=torch.long, device="cuda"), bias_id=torch.zeros(0, dtype=torch.int32, device="cuda"),
             bias=torch.zeros(0, device="cuda"))
    check_fwd(c)


@pytest.mark.parametrize("over", [False, True])
def test_many_biases_of_few_tokens_are_added_in_their_order(over):
    # sums that depend on the order, the same in every run
    V, n = 5000, 700
    z = torch.zeros(2, V, device="cuda")
    g = torch.Generator().manual_seed(7)
    ids = torch.randint(0, 3, (2 * n,), generator=g).to(torch.int32)
    b = torch.randn(2 * n, generator=g) * 10.0 ** torch.randint(-3, 5, (2 * n,), generator=g)
    L = B.make_logits(z)
    A = B.make_adjust(L, bias_start=torch.tensor([0, n, 2 * n], device="cuda"), bias_id=ids.cuda(), bias=b.cuda())
    out = z if over else torch.empty_like(z)
    B.oapl_logits_adjust(L, A, out)
    want = torch.zeros(2, V)
    for i in range(2 * n):
        want[i // n, ids[i]] = want[i // n, ids[i]] + b[i]
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("V", [2000, 2001])
def test_infinities_nan_and_lowest_values(V):
    c = make(8, V, "f32", 8)
    g = torch.Generator(device="cuda").manual_seed(2)
    for v in (math.inf, -math.inf, math.nan, torch.finfo(torch.float32).min, 0.0, -0.0):
        c["z"][torch.rand(8, V, device="cuda", generator=g) < 0.05] = v
    z = c["z"].clone()
    count, seen, bias, size, open_ = parts(c)
    L = B.make_logits(c["z"])
    out = torch.empty_like(z)
    B.oapl_logits_adjust(L, args(L, c), out)
    quiet = open_ & ~seen & (size == 0)
    assert torch.equal(out[quiet].view(torch.int32), z[quiet].view(torch.int32))      # NaN and -0 bit for bit
    assert bool((out[~open_] == -math.inf).all())
    assert torch.equal(torch.isnan(out), torch.isnan(z) & open_)
    inf = torch.isinf(z) & open_
    assert torch.equal(out[inf], z[inf])
    # a gradient that is not finite does not pass the mask
    d = torch.full_like(z, math.nan)
    B.oapl_logits_adjust_bwd(L, args(L, c), d, d)
    assert bool((d[~open_] == 0).all()) and bool(torch.isnan(d[open_]).all())


def test_rows_of_a_mask_by_index():
    c = make(7, 1000, "bf16", 9, allowed=0.5)
    table = c["open"][:3].clone()
    table[1] = False
    which = torch.tensor([2, -1, 0, 0, 1, -5, 2], dtype=torch.int32, device="cuda")
    c["open"] = torch.where((which >= 0)[:, None], table[which.long().clamp(min=0)], torch.tensor(True, device="cuda"))
    c["allowed"], c["allowed_row"] = pack(table), which
    check_fwd(c)
    check_bwd(c)
    wide = torch.full((3, 40), -1, dtype=torch.int32, device="cuda")
    wide[:, :32] = pack(table)
    c["allowed"] = wide[:, :35]         # rows of words some way apart
    check_fwd(c)


def test_what_only_the_device_can_see():
    c = make(5, 600, "bf16", 10, bias=4, allowed=None)
    T = c["tokens"].numel()
    for bad in ([-1, 2, 3], [3, 2, 4], [3, 5, 4], [0, 1, T + 1]):
        e = dict(c, spans=c["spans"].clone())
        e["spans"][3] = torch.tensor(bad)
        clean = dict(e, spans=e["spans"].clone())
        clean["spans"][3] = 0
        L = B.make_logits(c["z"])
        want, got, st = torch.empty_like(c["z"]), torch.empty_like(c["z"]), torch.zeros(1, dtype=torch.int32, device="cuda")
        B.oapl_logits_adjust(L, args(L, clean), want)
        B.oapl_logits_adjust(L, args(L, e), got, st)
        assert torch.equal(want, got) and int(st) == -6
        st.zero_()
        B.oapl_logits_adjust_bwd(L, args(L, e), got.clone(), got, st)
        assert int(st) == -6
    for bad in (-1, 10 ** 9):
        e = dict(c, bias_start=c["bias_start"].clone())
        e["bias_start"][2] = bad
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        L = B.make_logits(c["z"])
        B.oapl_logits_adjust(L, args(L, e), torch.empty_like(c["z"]), st)
        assert int(st) == -6
    c = make(5, 600, "bf16", 11)
    c["allowed_row"] = torch.tensor([0, 1, 5, 3, 4], dtype=torch.int32, device="cuda")
    c["open"][2] = True
    check_fwd(c, status=-5)


def test_row_offsets_beyond_32_bits():
    N, V = 29000, 152064        # 4.4e9 elements
    z = torch.empty(N, V, dtype=torch.bfloat16, device="cuda").fill_(1.0)
    toks = torch.tensor([5, 5, 152063], dtype=torch.int32, device="cuda")
    spans = torch.zeros(N, 3, dtype=torch.long, device="cuda")
    spans[:, 2] = 3
    L = B.make_logits(z)
    A = B.make_adjust(L, toks, spans, frequency=torch.full((N,), 0.5, device="cuda"))
    B.oapl_logits_adjust(L, A, z)
    for n in (0, 14122, 14123, 28245, N - 1):
        assert float(z[n, 5]) == 0.0 and float(z[n, 152063]) == 0.5 and float(z[n].float().sum()) == V - 1.5
    assert bool((z[:, 5] == 0).all()) and bool((z[:, 152063] == 0.5).all())


def test_gradient_over_its_input_and_over_the_logits():
    for V in (1000, 5001):
        c = make(6, V, "bf16", 12)
        check_bwd(c, where="d")
        check_bwd(c, where="z")


def test_gradient_is_that_of_the_adjustment():
    # piecewise linear: differences along a direction that crosses no zero are exact up to rounding
    V = 500
    c = make(4, V, "f32", 13)
    z = torch.where(c["z"].abs() < 0.5, torch.tensor(0.75, device="cuda"), c["z"])
    step = 0.25 * torch.rand(4, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    w = torch.randn(4, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    outs = []
    for x in (z, z + step):
        L = B.make_logits(x)
        o = torch.empty_like(x)
        B.oapl_logits_adjust(L, args(L, c), o)
        outs.append(torch.where(c["open"], o, 0.0).double())
    L = B.make_logits(z)
    dz = torch.empty_like(z)
    B.oapl_logits_adjust_bwd(L, args(L, c), w, dz)
    diff, along = (outs[1] - outs[0]) * w.double(), dz.double() * step.double()
    assert bool(((diff - along).abs() <= 8 * U * (outs[0].abs() + outs[1].abs() + 8) * w.double().abs()).all())


def test_other_stream_two_calls_at_once_and_captured():
    c = make(64, 30000, "bf16", 14, prompt=500, answer=500)
    L = B.make_logits(c["z"])
    A = args(L, c)
    want = torch.empty_like(c["z"])
    B.oapl_logits_adjust(L, A, want)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want) for _ in range(2)]
    for s, o in zip(streams, outs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(5):
                B.oapl_logits_adjust(L, A, o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        with torch.cuda.graph(graph, stream=streams[0]):
            B.oapl_logits_adjust(L, A, outs[0])
        for _ in range(3):
            outs[0].zero_()
            graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)


def test_together_with_the_log_probabilities_and_their_gradient():
    # adjust -> logprobs -> their gradient -> the adjustment's gradient, against automatic differentiation in 64 bits
    N, V = 12, 3000
    c = make(N, V, "f32", 15, allowed=0.8)
    c["open"][1] = c["open"][2]
    targets = torch.stack([torch.nonzero(r)[k, 0] for k, r in enumerate(c["open"])]).to(torch.int32)
    c["allowed"] = pack(c["open"])
    L = B.make_logits(c["z"])
    A = args(L, c)
    adj = torch.empty_like(c["z"])
    B.oapl_logits_adjust(L, A, adj)
    La = B.make_logits(adj, targets)
    lp, ent, lse = (torch.empty(N, device="cuda") for _ in range(3))
    B.oapl_logits_logprobs(La, lp, ent, lse)
    g1, g2 = torch.randn(N, device="cuda"), torch.randn(N, device="cuda")
    B.oapl_logits_logprobs_bwd(La, lse, ent, g1, g2, None, None, adj)
    dz = torch.empty_like(adj)
    B.oapl_logits_adjust_bwd(L, A, adj, dz)

    count, seen, bias, _, open_ = parts(c)
    z = c["z"].double().requires_grad_()
    r, f, p = row(c, "repetition", 1.0), row(c, "frequency", 0.0), row(c, "presence", 0.0)
    a = torch.where(seen, torch.where(z > 0, z / r, z * r), z) - f * count - p * (count > 0) + bias
    a = a.masked_fill(~open_, -1e300)
    ln_p = torch.log_softmax(a, 1)
    want_lp = ln_p.gather(1, targets.long()[:, None])[:, 0]
    want_ent = -(ln_p.exp() * ln_p).masked_fill(~open_, 0.0).sum(1)
    assert float((lp.double() - want_lp.detach()).abs().max()) < 1e-4 and float((ent.double() - want_ent.detach()).abs().max()) < 1e-4
    (g1.double() * want_lp + g2.double() * want_ent).sum().backward()
    # fp32 sums over the vocabulary and |lse| 2^-24 of each probability: within 1e-4 of the largest gradient
    assert float((dz.double() - z.grad).abs().max()) <= 1e-4 * float(z.grad.abs().max())


def test_binding_refusals():
    z = torch.zeros(4, 100, device="cuda")
    L = B.make_logits(z)
    toks, spans = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, dtype=torch.long, device="cuda")
    bits = torch.zeros(4, 4, dtype=torch.int32, device="cuda")
    for bad in (lambda: B.make_adjust(L, toks.long(), spans), lambda: B.make_adjust(L, toks, spans[:3]),
                lambda: B.make_adjust(L, toks, spans.int()), lambda: B.make_adjust(L, toks, spans, torch.ones(3, device="cuda")),
                lambda: B.make_adjust(L, allowed=bits[:3]), lambda: B.make_adjust(L, allowed=bits[:, :3]),
                lambda: B.make_adjust(L, allowed=bits.long()),
                lambda: B.oapl_logits_adjust(L, B.make_adjust(L), z.half()), lambda: B.oapl_logits_adjust(L, B.make_adjust(L), z[:3])):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_logits_adjust(L, B.make_adjust(L, toks), z)
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_logits_adjust(L, B.make_adjust(L, repetition=torch.ones(4, device="cuda")), z)
