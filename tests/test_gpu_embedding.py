"""oapl_embedding and its gradient against plain 64-bit forms of the same definitions."""
import pytest
import torch

from paper_2602_19362_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24      # half a step of fp32


def half_step(want, t):
    """Half a step of type t at `want`, also below its normal numbers."""
    f = torch.finfo(t)
    return want.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def rand(g, rows, cols, t, pad=0, offset=0, std=1.0):
    flat = torch.randn(rows * (cols + pad) + offset, device="cuda", generator=g).mul_(std).to(TYPES[t])
    return flat[offset:].view(rows, cols + pad)[:, :cols]


def ids_of(g, N, V, kind):
    if kind == "one":
        return torch.full((N,), V - 1, dtype=torch.int32, device="cuda")
    if kind == "rank":      # a token's share falls with its rank, as in text
        u = torch.rand(N, device="cuda", generator=g, dtype=torch.float64)
        return ((V ** u).long() - 1).clamp(0, V - 1).to(torch.int32)
    return torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)


def check_fwd(N, V, d, ti, to, scale, seed, pad=0, offset=0, masked=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = rand(g, V, d, ti, pad, offset)
    ids = ids_of(g, N, V, "any")
    mask = (torch.rand(N, device="cuda", generator=g) < 0.8).to(torch.uint8) if masked else None
    if masked:
        ids = torch.where(mask.bool(), ids, torch.tensor(-7, dtype=torch.int32, device="cuda"))
    whole = torch.full((N, d + pad + 16), 7.0, dtype=TYPES[to], device="cuda")
    out = whole[:, :d]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_embedding(B.make_lookup(ids, V, mask, scale), table, out, st)
    want = table[ids.long().clamp(min=0)].double() * torch.tensor(scale, dtype=torch.float32).item()
    if masked:
        want = torch.where(mask.bool()[:, None], want, 0.0)
    assert bool(((out.double() - want).abs() <= half_step(want, TYPES[to]) + 1.1 * U * want.abs()).all())
    assert bool((whole[:, d:] == 7.0).all()) and int(st) == 0
    if scale == 1.0 and ti == to and not masked:
        assert torch.equal(out, table[ids.long()])


@pytest.mark.parametrize("ti,to", [(a, b) for a in TYPES for b in TYPES])
@pytest.mark.parametrize("d", [1, 7, 8, 64, 257, 1000, 3584])
def test_lookup_types_and_sizes(ti, to, d):
    check_fwd(1, 3, d, ti, to, 1.0, d, masked=False)
    check_fwd(37, 1001, d, ti, to, 31.6, d + 1)
    check_fwd(130, 50, d, ti, to, 1.0, d + 2, pad=3, offset=1)


def test_lookup_many_rows():
    for N, d, pad in [(20001, 1536, 0), (5003, 1001, 2), (100000, 64, 0)]:
        check_fwd(N, 50021, d, "bf16", "bf16", 1.0, N, pad)


def test_lookup_keeps_what_is_not_finite_and_reports_ids_outside():
    table = torch.randn(10, 16, device="cuda")
    table[3, 5], table[4, 6] = float("inf"), float("nan")
    ids = torch.tensor([3, 4, 10, -1, 2 ** 31 - 1, 9], dtype=torch.int32, device="cuda")
    out = torch.full((6, 16), 5.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.oapl_embedding(B.make_lookup(ids, 10), table, out, st)
    want = torch.cat([table[3:5], torch.zeros(3, 16, device="cuda"), table[9:]])
    assert torch.equal(out.view(torch.int32), want.view(torch.int32)) and int(st) == -5
    mask = torch.tensor([1, 1, 0, 0, 0, 1], dtype=torch.uint8, device="cuda")
    st.zero_()
    B.oapl_embedding(B.make_lookup(ids, 10, mask), table, out, st)
    assert torch.equal(out.view(torch.int32), want.view(torch.int32)) and int(st) == 0


def test_lookup_offsets_beyond_32_bits():
    V, d = 600000, 4096
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    rows = [0, 524287, 524288, V - 1]       # around element 2^31
    for r in rows:
        table[r] = r % 251 + 1
    ids = torch.tensor(rows, dtype=torch.int32, device="cuda")
    out = torch.empty(4, d, dtype=torch.bfloat16, device="cuda")
    B.oapl_embedding(B.make_lookup(ids, V), table, out)
    assert torch.equal(out, table[ids.long()])


# ------------------------------------------------------------------------------------------------ gradient

def workspace(N, V, d):
    return torch.full((B.oapl_embedding_workspace_bytes(N, V, d),), 0xFF, dtype=torch.uint8, device="cuda")


def ref_bwd(ids, mask, dout, V, scale, old):
    live = torch.ones(ids.shape[0], dtype=torch.bool, device="cuda") if mask is None else mask.bool()
    at = live & (ids >= 0) & (ids < V)
    x = dout[at].double()
    total = torch.zeros(V, dout.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids[at].long(), x)
    size = torch.zeros_like(total).index_add_(0, ids[at].long(), x.abs())
    count = torch.bincount(ids[at].long(), minlength=V).double()[:, None]
    want = total * scale + (0 if old is None else old.double())
    # a sum of m terms in any fixed order is off by at most m - 1 half steps of the terms' magnitudes; the scale is one
    # rounding more, adding the old value another
    tol = count * U * size * abs(scale) + 2 * U * (want.abs() + size * abs(scale))
    return want, tol, count[:, 0]


def check_bwd(N, V, d, t, kind="any", scale=1.0, accumulate=False, pad=0, offset=0, masked=False, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + N)
    ids = ids_of(g, N, V, kind)
    mask = (torch.rand(N, device="cuda", generator=g) < 0.7).to(torch.uint8) if masked else None
    if masked:
        ids = torch.where(mask.bool(), ids, torch.tensor(-1, dtype=torch.int32, device="cuda"))
    dout = rand(g, N, d, t, pad, offset)
    whole = torch.randn(V, d + pad, device="cuda", generator=g)
    before = whole.clone()
    table = whole[:, :d]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = torch.tensor(scale, dtype=torch.float32).item()
    B.oapl_embedding_bwd(B.make_lookup(ids, V, mask, scale), dout, table, accumulate, workspace(N, V, d), st)
    want, tol, count = ref_bwd(ids, mask, dout, V, scale, before[:, :d] if accumulate else None)
    off = (table.double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())
    assert torch.equal(whole[:, d:], before[:, d:]) and int(st) == 0
    if accumulate:      # rows without a token are not touched
        assert torch.equal(table[count == 0], before[:, :d][count == 0])
    else:
        assert bool((table[count == 0] == 0).all())
    return table


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("N,V,d,pad,offset", [(1, 1, 1, 0, 0), (1, 1000, 64, 0, 0), (3, 2, 7, 1, 0), (31, 40, 8, 0, 0),
                                              (32, 5, 16, 8, 0), (33, 33, 1000, 0, 1), (64, 64, 257, 3, 0), (1000, 300, 129, 0, 0),
                                              (1024, 200, 264, 0, 0), (1025, 200, 264, 0, 0), (700, 3001, 2056, 0, 0),
                                              (8192, 5000, 72, 0, 0), (8193, 5000, 72, 0, 0), (20011, 1023, 40, 0, 0),
                                              (20011, 1024, 33, 2, 1), (30000, 70001, 24, 0, 0)])
def test_gradient_sizes(t, N, V, d, pad, offset):
    check_bwd(N, V, d, t, "any", 1.0, False, pad, offset, False)
    check_bwd(N, V, d, t, "rank", 31.6, True, pad, offset, True)


@pytest.mark.parametrize("N", [33, 100, 1024, 1025, 8192, 8200, 70000, 300007])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_one_token_for_all_rows(N, accumulate):
    # a run over all chunks, joined by one CTA for each slab
    check_bwd(N, 3, 40, "bf16", "one", 1.0, accumulate)
    check_bwd(N, 152064, 16, "f32", "one", 0.5, accumulate, masked=True) if N < 1000 else None


def test_gradient_of_a_text_like_batch_with_wide_rows():
    check_bwd(40960, 20000, 1536, "bf16", "rank")
    check_bwd(9001, 3000, 3584, "f16", "rank", 2.0, True, masked=True)
    check_bwd(3001, 5021, 1001, "f16", "rank", 31.6, False, pad=2, masked=True)


@pytest.mark.parametrize("N", [1105, 1156, 1190, 4913, 8177, 8211, 20230])
def test_gradient_writes_the_last_tokens_of_the_list(N):
    # every row of the table has a token, or all but one: what is cleared lies between the ends that a search finds
    V, d = -(-N // 5), 8
    ids = torch.arange(N, device="cuda", dtype=torch.int32) // 5
    for gone in (None, 0, 31, 32, V // 2, V - 1):
        keep = ids[ids != gone] if gone is not None else ids
        dout = torch.ones(keep.numel(), d, device="cuda")
        table = torch.full((V, d), 7.0, device="cuda")
        B.oapl_embedding_bwd(B.make_lookup(keep, V), dout, table, False, workspace(keep.numel(), V, d))
        want = torch.bincount(keep.long(), minlength=V).float()[:, None].expand(V, d)
        assert torch.equal(table, want), gone


def test_gradient_runs_that_begin_and_end_at_chunks():
    # runs of 32, 31, 33, 64 and 1 rows in every alignment to the chunks of 32
    lens = [32, 32, 31, 1, 33, 31, 64, 1, 1, 62, 128, 5, 27, 32, 1]
    ids = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).to(torch.int32).cuda()
    ids = ids[torch.randperm(ids.numel(), generator=torch.Generator().manual_seed(3)).cuda()]
    N, V, d = ids.numel(), len(lens) + 2, 24
    dout = torch.randint(-8, 9, (N, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()
    table = torch.full((V, d), 3.0, device="cuda")
    B.oapl_embedding_bwd(B.make_lookup(ids, V), dout, table, False, workspace(N, V, d))
    want = torch.zeros(V, d, device="cuda").index_add_(0, ids.long(), dout)
    assert torch.equal(table, want)         # whole numbers: exact in any order


def test_gradient_without_any_row_that_counts():
    N, V, d = 50, 70, 24
    ids = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    dout = torch.full((N, d), float("nan"), device="cuda")
    for mask, status in [(torch.zeros(N, dtype=torch.uint8, device="cuda"), 0), (None, -5)]:
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        table = torch.ones(V, d, device="cuda")
        B.oapl_embedding_bwd(B.make_lookup(ids, V, mask), dout, table, True, workspace(N, V, d), st)
        assert bool((table == 1).all()) and int(st) == status
        B.oapl_embedding_bwd(B.make_lookup(ids, V, mask), dout, table, False, workspace(N, V, d), st)
        assert bool((table == 0).all())


def test_gradient_ids_outside_count_for_nothing():
    for N in (500, 2000, 9000):
        g = torch.Generator(device="cuda").manual_seed(N)
        V, d = 64, 16
        ids = torch.randint(-5, V + 5, (N,), device="cuda", generator=g).to(torch.int32)
        dout = rand(g, N, d, "f32")
        dout[(ids < 0) | (ids >= V)] = float("inf")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        table = torch.full((V, d), 9.0, device="cuda")
        B.oapl_embedding_bwd(B.make_lookup(ids, V), dout, table, False, workspace(N, V, d), st)
        want, tol, _ = ref_bwd(ids, None, dout, V, 1.0, None)
        assert bool(((table.double() - want).abs() <= tol).all()) and int(st) == -5


def test_gradient_repeats_bit_for_bit():
    g = torch.Generator(device="cuda").manual_seed(5)
    for N in (900, 5000, 50000):
        ids, dout = ids_of(g, N, 3000, "rank"), rand(g, N, 256, "bf16")
        got = []
        for _ in range(3):
            table = torch.empty(3000, 256, device="cuda")
            B.oapl_embedding_bwd(B.make_lookup(ids, 3000), dout, table, False, workspace(N, 3000, 256))
            got.append(table)
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_gradient_is_that_of_the_lookup():
    # sum(w * lookup(table)) is linear in the table: its difference quotient is exact up to rounding
    g = torch.Generator(device="cuda").manual_seed(8)
    N, V, d, s = 300, 50, 24, 2.0
    table, w, step = (rand(g, r, d, "f32") for r in (V, N, V))
    ids = ids_of(g, N, V, "any")
    k = B.make_lookup(ids, V, scale=s)
    out = [torch.empty(N, d, device="cuda") for _ in range(2)]
    B.oapl_embedding(k, table, out[0])
    B.oapl_embedding(k, table + step, out[1])
    grad = torch.empty(V, d, device="cuda")
    B.oapl_embedding_bwd(k, w, grad, False, workspace(N, V, d))
    diff = ((out[1].double() - out[0].double()) * w.double()).sum()
    want = (grad.double() * step.double()).sum()
    # table + step, its scaled value and the difference: a few half steps of each of the N d products' factors
    tol = 8 * U * ((table.abs().max() + step.abs().max()) * s * w.abs().sum()).double()
    assert float((diff - want).abs()) <= float(tol)


def test_other_stream_and_captured_graphs_that_share_a_workspace():
    g = torch.Generator(device="cuda").manual_seed(11)
    N, V, d = 9000, 2000, 128
    ids, dout = ids_of(g, N, V, "rank"), rand(g, N, d, "bf16")
    other = ids_of(g, 700, V, "any")
    ws = workspace(N, V, d)
    want = torch.empty(V, d, device="cuda")
    want2 = torch.empty(V, d, device="cuda")
    B.oapl_embedding_bwd(B.make_lookup(ids, V), dout, want, False, ws)
    B.oapl_embedding_bwd(B.make_lookup(other, V), dout[:700], want2, False, ws)
    got, got2 = torch.empty(V, d, device="cuda"), torch.empty(V, d, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.stream(side):
        with torch.cuda.graph(graphs[0], stream=side):
            B.oapl_embedding_bwd(B.make_lookup(ids, V), dout, got, False, ws)
        with torch.cuda.graph(graphs[1], stream=side):
            B.oapl_embedding_bwd(B.make_lookup(other, V), dout[:700], got2, False, ws)
        for _ in range(3):
            got.fill_(float("nan"))
            got2.fill_(float("nan"))
            graphs[0].replay()
            graphs[1].replay()
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got2, want2)


def test_binding_refusals():
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    k = B.make_lookup(ids, 10)
    table, out = torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    for bad in (lambda: B.make_lookup(ids.long(), 10), lambda: B.make_lookup(ids[::2], 10),
                lambda: B.make_lookup(ids, 10, torch.ones(4, device="cuda")),
                lambda: B.oapl_embedding(k, table[:9], out), lambda: B.oapl_embedding(k, table, out[:3]),
                lambda: B.oapl_embedding(k, table, out[:, :7]), lambda: B.oapl_embedding(k, table.double(), out),
                lambda: B.oapl_embedding(k, table.t().contiguous().t(), out),
                lambda: B.oapl_embedding_bwd(k, out, table.half(), False, workspace(4, 10, 8)),
                lambda: B.oapl_embedding_bwd(k, out, table, False, torch.zeros(4096, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(B.OaplError, match="WORKSPACE_TOO_SMALL"):
        B.oapl_embedding_bwd(k, out, table, False, torch.zeros(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_embedding(k, table, table[:4])
    with pytest.raises(B.OaplError, match="INVALID_ARG"):
        B.oapl_embedding(B.make_lookup(ids[:0], 10), table, out[:0])
