"""oapl_quantize and oapl_scaled_matmul against plain forms: quantisation bit for bit, the product in 64 bits."""
import math

import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
FLOOR = 2.0 ** -100


def blocks(x, b):
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, (-c) % 128, 0, (-r) % b))
    return x.view(x.shape[0] // b, b, x.shape[1] // 128, 128)


def ref_quantize(x, to, b, turn, pow2):
    """The definition, in fp32 with IEEE division as the scale is stored."""
    x = x.float()
    x = x.t().contiguous() if turn else x
    rows, cols = x.shape
    xb = blocks(x, b)
    amax = xb.abs().amax((1, 3)).clamp_min(FLOOR)
    top = TOP[to]
    if pow2:
        # smallest power of two that is at least amax / top
        m, e = torch.frexp(amax.double() / top)
        scale = torch.ldexp(torch.ones_like(m), torch.where(m == 0.5, e - 1, e)).float()
        q = xb / scale[:, None, :, None]
    else:
        scale = (amax.double() / top).float()      # a tensor over a number would be multiplied by its reciprocal
        q = (xb * 0.875) / (amax * (0.875 / top))[:, None, :, None]
    q = q.flatten(2).flatten(0, 1)[:rows, :cols]
    return q.clamp(-top, top).to(F8[to]), scale


def alloc(rows, cols, b, to, pad=0):
    ld = -(-cols // 16) * 16 + 16 * pad
    store = torch.full((rows, ld), 0x5A, dtype=torch.uint8, device="cuda")
    data = store.view(F8[to])[:, :cols]
    scale = torch.full((-(-cols // 128), -(-rows // b)), -9.0, device="cuda").t()
    return store, B.make_scaled(data, scale, b)


def check_quantize(x, to, b, turn, pow2, pad=0):
    rows, cols = x.shape[::-1] if turn else x.shape
    store, out = alloc(rows, cols, b, to, pad)
    B.oapl_quantize(x, out, turn, pow2)
    q, scale = ref_quantize(x, to, b, turn, pow2)
    got_q, got_s = out.tensors
    assert torch.equal(torch.nan_to_num(got_s, nan=-1.0), torch.nan_to_num(scale, nan=-1.0))
    gf, wf = got_q.float(), q.float()
    assert torch.equal(torch.isnan(gf), torch.isnan(wf))
    assert torch.equal(torch.nan_to_num(gf), torch.nan_to_num(wf))
    assert bool((store[:, cols:] == 0x5A).all())       # the padding behind a row stays


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("to", ["e4m3", "e5m2"])
@pytest.mark.parametrize("b", [1, 128])
@pytest.mark.parametrize("turn", [False, True])
def test_quantize_sizes(t, to, b, turn):
    g = torch.Generator(device="cuda").manual_seed(3)
    for R, C, ld, off in [(1, 1, 1, 0), (1, 129, 129, 0), (5, 16, 24, 0), (128, 128, 128, 0), (130, 257, 257, 1),
                          (127, 384, 384, 0), (300, 1000, 1003, 3), (513, 136, 136, 0)]:
        flat = torch.randn(R * ld + off, device="cuda", generator=g).mul_(torch.exp(torch.randn(1, device="cuda", generator=g) * 3)).to(TYPES[t])
        x = flat[off:].view(R, ld)[:, :C]
        for pow2 in (False, True):
            check_quantize(x, to, b, turn, pow2, pad=1 if R == 5 else 0)


@pytest.mark.parametrize("b", [1, 128])
@pytest.mark.parametrize("turn", [False, True])
@pytest.mark.parametrize("pow2", [False, True])
def test_quantize_zeros_extremes_nan_inf(b, turn, pow2):
    x = torch.randn(512, 512, device="cuda")
    x[0:128, 0:128] = 0.0
    x[128:256, 0:128] *= 1e-37                     # below the floor of a block's magnitude
    x[256:384, 0:128] *= 1e37
    x[0, 200] = 448.0                              # exactly the largest value: scale 1
    x[130, 200] = 57344.0
    check_quantize(x, "e4m3", b, turn, pow2)
    check_quantize(x, "e5m2", b, turn, pow2)
    x[5, 130] = math.nan
    x[200, 300] = math.inf
    x[201, 301] = -math.inf
    check_quantize(x, "e4m3", b, turn, False)
    check_quantize(x.to(torch.bfloat16), "e5m2", b, turn, False)


def test_quantize_rounds_half_way_values_to_even():
    # 16 j + 8 with a scale of 1 lies half way between two e4m3 values above 128
    x = torch.zeros(1, 128, device="cuda", dtype=torch.bfloat16)
    x[0, 0] = 448.0
    x[0, 1:17] = torch.arange(16, device="cuda") * 16 + 136
    out = B.alloc_scaled(1, 128, 1)
    B.oapl_quantize(x, out)
    assert float(out.tensors[1][0, 0]) == 1.0
    want = x.float().to(torch.float8_e4m3fn).float()
    assert torch.equal(out.tensors[0].float(), want)


def test_quantize_offsets_beyond_32_bits():
    R, C = 18000, 131072      # 2.36e9 values
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    x[R - 1] = torch.randn(C, device="cuda").to(torch.bfloat16)
    out = B.alloc_scaled(R, C, 1)
    B.oapl_quantize(x, out)
    q, s = ref_quantize(x[R - 1:], "e4m3", 1, False, False)
    assert torch.equal(out.tensors[0][R - 1:].float(), q.float()) and torch.equal(out.tensors[1][R - 1:], s)
    del out
    out = B.alloc_scaled(C, R, 1)
    B.oapl_quantize(x, out, transpose=True)
    assert torch.equal(out.tensors[0][:, :128].float().abs().sum(), torch.zeros((), device="cuda"))
    q, s = ref_quantize(x[R - R % 128:], "e4m3", 1, True, False)
    assert torch.equal(out.tensors[0][:, R - R % 128:].float(), q.float()) and torch.equal(out.tensors[1][:, -1:], s)


# ---------------------------------------------------------------------------------------- product

def rand_scaled(rows, cols, b, to, seed, layout="k"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = -(-cols // 16) * 16
    # what lies behind a row must not count: NaN
    store = torch.full((rows, ld), 0x7F, dtype=torch.uint8, device="cuda").view(F8[to])
    data = store[:, :cols]
    data.copy_((torch.randn(rows, cols, device="cuda", generator=g) * (TOP[to] / 4)).clamp(-TOP[to], TOP[to]).to(F8[to]))
    rb, kb = -(-rows // b), -(-cols // 128)
    s = torch.rand(rb, kb, device="cuda", generator=g).add_(0.5).mul_(4.0 / TOP[to])
    s *= torch.exp(torch.randn(1, kb, device="cuda", generator=g))
    if layout == "k":
        scale = torch.empty(kb, rb, device="cuda").t().copy_(s)
    elif layout == "row":
        scale = s.contiguous()
    elif layout == "wide":
        scale = torch.full((rb, 3 * kb), math.nan, device="cuda")[:, ::3].copy_(s)
    else:       # one scale for all rows of a column block
        scale = s[:1].expand(rb, kb)
    return B.make_scaled(data, scale, b)


def widen(m):
    data, scale = m.tensors
    x = data.double()
    s = scale.double().repeat_interleave(m.block_rows, 0)[:x.shape[0]].repeat_interleave(128, 1)[:, :x.shape[1]]
    return x * s


def check_matmul(A, W, out, ldc_pad=0, accumulate=False, offset=0):
    M, N, K = A.rows, W.rows, A.cols
    t = TYPES[out]
    flat = torch.full((M * (N + ldc_pad) + offset,), 3.0, dtype=t, device="cuda")
    C = flat[offset:].view(M, N + ldc_pad)[:, :N]
    old = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    if accumulate:
        C.normal_()
        old = C.double()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_scaled_matmul(A, W, C, accumulate, st)
    assert int(st) == 0
    a, b = widen(A), widen(W)
    want = a @ b.t() + old
    size = a.abs() @ b.abs().t()
    # one rounding to the type; nk fp32 additions of scaled blocks with two more roundings each; inside a block
    # four instructions of 32 exact products, whose sums keep at least 2^-23 of their largest term each
    nk = -(-K // 128)
    tol = torch.finfo(t).eps / 2 * want.abs() + size * (nk + 3 + 4 * 33) * 2.0 ** -23 + old.abs() * 2.0 ** -23
    tol = tol + torch.finfo(t).smallest_normal * torch.finfo(t).eps
    bad = (C.double() - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), C[bad][:4], want[bad][:4])
    # and on average far closer than that: no block goes missing
    rel = float((C.double() - want).norm() / want.norm())
    assert rel <= torch.finfo(t).eps / 2 + 1e-5, rel
    if ldc_pad:
        assert bool((flat[offset:].view(M, N + ldc_pad)[:, N:] == 3.0).all())
    assert bool((flat[:offset] == 3.0).all())
    return C


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bb", [128, 1])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 1000, 128), (3, 130, 300), (16, 512, 64), (100, 129, 257), (128, 256, 1024),
                                   (257, 255, 640), (300, 1000, 1999), (600, 777, 130)])
def test_matmul_sizes(out, bb, M, N, K):
    A, W = rand_scaled(M, K, 1, "e4m3", M + N), rand_scaled(N, K, bb, "e4m3", K)
    check_matmul(A, W, out)


@pytest.mark.parametrize("ta,tb", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
def test_matmul_types(ta, tb):
    check_matmul(rand_scaled(300, 500, 1, ta, 1), rand_scaled(400, 500, 128, tb, 2), "f32")
    check_matmul(rand_scaled(20, 500, 1, ta, 1), rand_scaled(400, 500, 1, tb, 2), "bf16")


@pytest.mark.parametrize("ba,bb", [(1, 1), (1, 128), (128, 1), (128, 128)])
@pytest.mark.parametrize("layout", ["k", "row", "wide", "one"])
def test_matmul_scale_layouts(ba, bb, layout):
    for M in (5, 290):
        check_matmul(rand_scaled(M, 900, ba, "e4m3", 3, layout), rand_scaled(520, 900, bb, "e4m3", 4, layout), "f32")


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (7, 3), (16, 0)])
def test_matmul_result_layout_and_accumulation(out, pad, offset):
    for M in (7, 270):
        A, W = rand_scaled(M, 384, 1, "e4m3", 5), rand_scaled(512, 384, 128, "e4m3", 6)
        check_matmul(A, W, out, pad, False, offset)
        check_matmul(A, W, out, pad, True, offset)
        check_matmul(A, rand_scaled(511, 384, 1, "e4m3", 7), out, pad, True, offset)


@pytest.mark.parametrize("M", [1, 8, 16, 17, 32, 33, 64, 65, 96, 128, 129, 256])
def test_matmul_few_rows(M):
    for N, K in [(4096, 2048), (5000, 3600), (1500, 200)]:
        A = rand_scaled(M, K, 1, "e4m3", M)
        check_matmul(A, rand_scaled(N, K, 128, "e4m3", N), "bf16")
        check_matmul(A, rand_scaled(N, K, 1, "e5m2", N), "f32")


def test_matmul_more_tiles_than_sms_and_long_k():
    check_matmul(rand_scaled(3000, 700, 1, "e4m3", 1), rand_scaled(5000, 700, 128, "e4m3", 2), "bf16")
    check_matmul(rand_scaled(5100, 140, 1, "e4m3", 1), rand_scaled(2900, 140, 1, "e4m3", 2), "f32")
    check_matmul(rand_scaled(200, 70000, 1, "e4m3", 1), rand_scaled(300, 70000, 128, "e4m3", 2), "f32")
    check_matmul(rand_scaled(9, 70001, 1, "e4m3", 1), rand_scaled(300, 70001, 128, "e4m3", 2), "f32")


def test_matmul_scales_of_nan_and_zero_stay_in_their_block():
    A, W = rand_scaled(200, 512, 1, "e4m3", 1), rand_scaled(384, 512, 128, "e4m3", 2)
    A.tensors[1][7, 2] = math.nan
    W.tensors[1][1, 1] = 0.0
    C = torch.empty(200, 384, device="cuda")
    B.oapl_scaled_matmul(A, W, C)
    assert bool(torch.isnan(C[7]).all()) and int(torch.isnan(C).sum()) == 384
    A.tensors[1][7, 2] = 1.0
    check_matmul(A, W, "f32")


def test_matmul_repeats_bit_for_bit_and_on_two_streams():
    pairs = [(rand_scaled(700, 1000, 1, "e4m3", 1), rand_scaled(900, 1000, 128, "e4m3", 2)),
             (rand_scaled(5, 1000, 1, "e4m3", 3), rand_scaled(900, 1000, 128, "e4m3", 4))]
    want = [check_matmul(a, w, "f32") for a, w in pairs]
    torch.cuda.synchronize()
    outs = []
    for a, w in pairs:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(10):
                C = torch.empty(a.rows, w.rows, device="cuda")
                B.oapl_scaled_matmul(a, w, C)
            outs.append(C)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_captured_and_replayed():
    x, w = torch.randn(300, 700, device="cuda"), torch.randn(500, 700, device="cuda").to(torch.bfloat16)
    A, W = B.alloc_scaled(300, 700, 1), B.alloc_scaled(500, 700, 128)
    few = B.alloc_scaled(9, 700, 1)
    C, D = torch.zeros(300, 500, device="cuda"), torch.zeros(9, 500, dtype=torch.bfloat16, device="cuda")

    def step():
        B.oapl_quantize(x, A)
        B.oapl_quantize(x[:9], few)
        B.oapl_quantize(w, W)
        B.oapl_scaled_matmul(A, W, C)
        B.oapl_scaled_matmul(few, W, D)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.normal_()
    graph.replay()
    torch.cuda.synchronize()
    got = C.clone(), D.clone()
    C.zero_()
    D.zero_()
    step()
    assert torch.equal(got[0], C) and torch.equal(got[1], D)
    assert float((C.double() - widen(A) @ widen(W).t()).abs().max()) < 1e-3


def test_matmul_row_offsets_beyond_32_bits():
    # the last rows of the weight, and of the result, start past 2^31 bytes and elements
    N, K = 18000, 131072
    W = B.make_scaled(torch.zeros(N, K, dtype=torch.uint8, device="cuda").view(F8["e4m3"]),
                      torch.ones(-(-N // 128), K // 128, device="cuda"), 128)
    W.tensors[0][N - 3:] = torch.randn(3, K, device="cuda").to(F8["e4m3"])
    for M in (2, 70):
        A = rand_scaled(M, K, 1, "e4m3", 1)
        C = torch.full((M, N), 7.0, device="cuda")
        B.oapl_scaled_matmul(A, W, C)
        want = widen(A) @ W.tensors[0][N - 3:].double().t()
        assert float((C[:, N - 3:].double() - want).abs().max()) <= 1e-5 * float(widen(A).abs().sum(1).max()) * 4
        assert bool((C[:, :N - 3] == 0).all())
    del W
    M, N = 70000, 32768
    C = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    A, W = rand_scaled(M, 128, 1, "e4m3", 1), rand_scaled(N, 128, 128, "e4m3", 2)
    B.oapl_scaled_matmul(A, W, C)
    want = widen(A)[-5:] @ widen(W).t()
    assert float((C[-5:].double() - want).norm() / want.norm()) < 2.0 ** -8
    assert not bool((C == 7.0).all(1).any())


def test_binding_refusals():
    A, W = rand_scaled(4, 256, 1, "e4m3", 1), rand_scaled(64, 256, 128, "e4m3", 2)
    with pytest.raises(TypeError):
        B.oapl_scaled_matmul(A, W, torch.empty(4, 65, device="cuda"))
    with pytest.raises(TypeError):
        B.oapl_scaled_matmul(A, W, torch.empty(4, 64, device="cuda", dtype=torch.float64))
    with pytest.raises(B.OaplError):
        B.oapl_scaled_matmul(A, rand_scaled(64, 240, 128, "e4m3", 2), torch.empty(4, 64, device="cuda"))
    with pytest.raises(ValueError):
        B.make_scaled(A.tensors[0], A.tensors[1], 64)
    with pytest.raises(TypeError):
        B.make_scaled(A.tensors[0], A.tensors[1][:3], 1)
    with pytest.raises(B.OaplError):            # rows not a multiple of 16 bytes apart
        B.oapl_scaled_matmul(B.make_scaled(torch.zeros(4, 100, dtype=torch.uint8, device="cuda").view(F8["e4m3"]),
                                           torch.ones(4, 1, device="cuda"), 1),
                             rand_scaled(64, 100, 128, "e4m3", 2), torch.empty(4, 64, device="cuda"))
    with pytest.raises(B.OaplError):            # turned, but out is not
        B.oapl_quantize(torch.zeros(4, 256, device="cuda"), A, transpose=True)


# ---------------------------------------------------------------------------------------- together

def test_head_in_eight_bits_forward_and_backward():
    """An 8-bit LM head as a trainer or an engine runs it: quantise H and W, logits, log-probabilities with
    entropy and alternatives, gradient of the logits, and dH, dW as 8-bit products; and the log-probabilities as
    the inference policy's side of the loss."""
    torch.manual_seed(0)
    N, d, V, S, P = 384, 512, 5003, 8, 2
    ldv = 5008
    H = torch.randn(N, d, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, d, device="cuda") / math.sqrt(d) * 2).to(torch.bfloat16)
    targets = torch.randint(0, V, (N,), device="cuda").to(torch.int32)
    mask = (torch.rand(N, device="cuda") < 0.9).to(torch.uint8)
    Hq, Wq = B.alloc_scaled(N, d, 1), B.alloc_scaled(V, d, 128)
    B.oapl_quantize(H, Hq)
    B.oapl_quantize(W, Wq)
    Z = torch.empty(N, ldv, dtype=torch.bfloat16, device="cuda")[:, :V]
    B.oapl_scaled_matmul(Hq, Wq, Z)
    L = B.make_logits(Z, targets, mask)
    lp, ent, lse = (torch.empty(N, device="cuda") for _ in range(3))
    top, ids = torch.empty(N, 5, device="cuda"), torch.empty(N, 5, dtype=torch.int32, device="cuda")
    B.oapl_logits_logprobs(L, lp, ent, lse, top, ids)

    # 64 bits, from the quantised matrices; a logit is off by at most half a bf16 step of itself, and a
    # log-probability by its own logit's error and a mean of the others'
    z = widen(Hq) @ widen(Wq).t()
    ref = torch.log_softmax(z, 1)
    live = mask.bool()
    half = 2.0 ** -9 * z.abs().amax(1) * 2
    assert bool(((lp - ref.gather(1, targets.long()[:, None])[:, 0]).abs()[live] <= (2 * half + 1e-4)[live]).all())
    assert bool((lp[~live] == 0).all())
    # 8-bit rounding of H and W leaves the bf16 head's log-probabilities near: e4m3 values are off by 2^-4 at most
    exact = torch.log_softmax(H.double() @ W.double().t(), 1).gather(1, targets.long()[:, None])[:, 0]
    assert float((lp - exact)[live].abs().mean()) < 0.2

    # gradient of sum(lp): dlogits, then both products
    dZ = torch.empty(N, ldv, dtype=torch.bfloat16, device="cuda")[:, :V]
    ones = torch.ones(N, device="cuda")
    B.oapl_logits_logprobs_bwd(L, lse, ent, ones, None, None, None, dZ)
    e5 = torch.float8_e5m2
    gq, gtq = B.alloc_scaled(N, V, 1, e5), B.alloc_scaled(V, N, 1, e5)
    Wt, Ht = B.alloc_scaled(d, V, 128), B.alloc_scaled(d, N, 1)
    B.oapl_quantize(dZ, gq)
    B.oapl_quantize(dZ, gtq, transpose=True)
    B.oapl_quantize(W, Wt, transpose=True)
    B.oapl_quantize(H, Ht, transpose=True)
    dH, dW = torch.empty(N, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(V, d, device="cuda")
    B.oapl_scaled_matmul(gq, Wt, dH)
    B.oapl_scaled_matmul(gtq, Ht, dW, accumulate=True)
    zz = z.clone().requires_grad_()
    (torch.log_softmax(zz, 1).gather(1, targets.long()[:, None])[:, 0] * live).sum().backward()
    want_H, want_W = zz.grad @ W.double(), zz.grad.t() @ H.double()
    # the one-hot term dominates: e5m2 is off by 2^-3 of a value at most, e4m3 by 2^-4; the norms of the
    # differences stay below the sum of both and the bf16 roundings
    lim = 2.0 ** -3 + 2.0 ** -4 + 2.0 ** -6
    assert float((dH.double() - want_H).norm() / want_H.norm()) < lim
    assert float((dW.double() - want_W).norm() / want_W.norm()) < lim
    # W turned in 128 x 128 blocks is the turned quantised W: same blocks, same scales
    assert torch.equal(Wt.tensors[0].float(), Wq.tensors[0].float().t()) and torch.equal(Wt.tensors[1], Wq.tensors[1].t())

    # the inference policy's log-probabilities as data of the loss
    seq_id = (torch.arange(N, device="cuda") // (N // S)).to(torch.int32)
    batch = dict(N=N, d=d, V=V, S=S, P=P, H=H, W=W, targets=targets, mask=mask, seq_id=seq_id,
                 group_id=(torch.arange(S, device="cuda") % P).to(torch.int32), reward=torch.ones(S, device="cuda"), logp_inf=lp)
    prob = B.make_problem(batch, 1.0, 1.0, 1.0 / S)
    ws = B.alloc_workspace(prob)
    loss, seq, vhat, delta = (torch.empty(n, device="cuda") for n in (1, S, P, S))
    B.oapl_loss_fwd(prob, loss, seq, vhat, delta, None, ws)
    assert B.oapl_get_last_status(ws) == 0
    D = torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, seq_id.long(), (exact - lp.double()) * live)
    assert float((delta.double() - D).abs().max()) <= 2e-3 * (N // S)       # all rewards equal: delta = D
