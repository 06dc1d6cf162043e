"""Cases for the operators between the token ids and the LM head, and between the LM head's logits and the sampler:

  embedding   rows of a table by token id, scaled; its gradient: rows of dout added up by token id
  residual    x' = a x + b gate * norm(y) and the next norm's h = norm(x'), as one step; its gradient
  adjust      penalties for repeated tokens, biases and a mask of allowed tokens on rows of logits; its gradient
  clip        the norm over a list of gradient tensors, and the list scaled to a largest norm

Each case is a dict with an "op" and, where the operator has one, "grad" for its backward pass. `own` selects what
`run` computes with: elementary torch operations, or the library's entry points.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # the tokens of a decode step of 64 requests
        dict(name="embedding decode", op="embedding", grad=False, N=64, V=152064, d=3584, ld=3584, type="bf16", to="bf16",
             scale=1.0, dead=0.0),
        # a packed training batch, its gradient into the weight that is also the LM head's (fp32, every row written)
        dict(name="embedding gradient", op="embedding", grad=True, N=40960, V=151936, d=1536, ld=1536, type="bf16",
             to="f32", scale=1.0, dead=0.0),
        # a small ragged batch: odd width, rows off 16-byte boundaries, padding, a scaled embedding
        dict(name="embedding gradient ragged", op="embedding", grad=True, N=3001, V=50021, d=1001, ld=1003, type="f16",
             to="f32", scale=31.6, dead=0.2),
        # the end of a block for eight decoded tokens
        dict(name="residual decode", op="residual", grad=False, N=8, d=5120, ld=5120, type="bf16", gate="none", post=True,
             weight="bf16"),
        # the same in training, with a gate per channel, and its gradient
        dict(name="residual training", op="residual", grad=False, N=16384, d=3584, ld=3584, type="bf16", gate="column",
             post=True, weight="bf16"),
        dict(name="residual gradient", op="residual", grad=True, N=16384, d=3584, ld=3584, type="bf16", gate="column",
             post=True, weight="bf16"),
        # odd width, fp32, a gate per element
        dict(name="residual gradient ragged", op="residual", grad=True, N=1531, d=1111, ld=1113, type="f32", gate="full",
             post=True, weight="f32"),
        # one request with a long prompt, all of the adjustments; the raw logits stay for the log-probabilities
        dict(name="adjust one request", op="adjust", grad=False, N=1, V=152064, ld=152064, type="f32", prompt=6000,
             output=2000, per=1, penal=True, bias=40, allowed=0.9, place="apart"),
        # a decode batch under a grammar that leaves a few tokens, over the logits themselves
        dict(name="adjust grammar", op="adjust", grad=False, N=64, V=128256, ld=128256, type="bf16", prompt=0, output=0,
             per=1, penal=False, bias=0, allowed=0.02, place="over"),
        # a trainer's chunk of rows whose sampler had penalties: the gradient of the raw logits
        dict(name="adjust gradient", op="adjust", grad=True, N=2048, V=152064, ld=152064, type="bf16", prompt=300,
             output=1024, per=1024, penal=True, bias=8, allowed=1.0, place="apart"),
        # the gradients of a model's blocks, left in bf16 by the backward pass, clipped into the optimizer's fp32 buffer
        dict(name="clip blocks", op="clip", d=1536, layers=12, small=0, type="bf16", to="f32", ratio=0.3),
        # hundreds of small tensors of odd sizes
        dict(name="clip small tensors", op="clip", d=0, layers=0, small=600, type="f32", to="f32", ratio=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embedding", "embedding", "residual", "residual", "adjust", "adjust", "clip"])
    type_ = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "embedding":
        grad = rng.random() < 0.5
        d = _log_int(rng, 64, 5120)
        d -= d % 8 if rng.random() < 0.7 else 0
        return dict(op=op, grad=grad, N=_log_int(rng, 1, min(65536, 120000000 // d)), V=_log_int(rng, 1000, min(152064, 500000000 // d)),
                    d=d, ld=d + rng.choice([0, 0, 8, 3]), type=type_, to="f32" if grad else rng.choice([type_, type_, "f32"]),
                    scale=rng.choice([1.0, 31.6]), dead=rng.choice([0.0, 0.0, 0.3]))
    if op == "residual":
        d = _log_int(rng, 64, 12288)
        d -= d % 8 if rng.random() < 0.7 else 0
        N = _log_int(rng, 1, min(100000, (58000000 if type_ != "f32" else 29000000) // d))
        return dict(op=op, grad=rng.random() < 0.5, N=N, d=d, ld=d + rng.choice([0, 0, 8, 1]), type=type_,
                    gate=rng.choice(["none", "row", "column", "full"]), post=rng.random() < 0.7, weight=rng.choice([type_, "f32"]))
    if op == "adjust":
        V = _log_int(rng, 1000, 152064)
        N = _log_int(rng, 1, min(8192, (2048 if type_ != "f32" else 1024) * 152064 // V))
        grad = rng.random() < 0.3
        output = _log_int(rng, 1, 4096)
        return dict(op=op, grad=grad, N=N, V=V, ld=V + rng.choice([0, (-V) % 8, rng.randint(1, 32)]), type=type_,
                    prompt=_log_int(rng, 1, 8000) if N <= 256 else _log_int(rng, 1, 500), output=min(output, 4096 if N <= 256 else 1024),
                    per=rng.choice([1, 64, 1024]), penal=rng.random() < 0.8, bias=rng.choice([0, 0, 3, 100]),
                    allowed=rng.choice([1.0, 0.9, 0.02]), place="apart")
    layers = rng.randint(0, 12)
    return dict(op=op, d=8 * _log_int(rng, 16, 192) if layers else 0, layers=layers, small=_log_int(rng, 1, 600), type=type_,
                to=rng.choice([type_, "f32"]), ratio=rng.choice([0.3, 0.9, 2.0]))


# ------------------------------------------------------------------------------------------------ inputs

def _normal(g, *shape, std=1.0, type_="f32", ld=None):
    """[rows, cols] with rows ld apart, or a vector."""
    if ld is None:
        return torch.empty(*shape, dtype=TYPES[type_], device="cuda").normal_(0.0, std, generator=g)
    return torch.empty(shape[0], ld, dtype=TYPES[type_], device="cuda").normal_(0.0, std, generator=g)[:, :shape[1]]


def _ids(g, n, V):
    """Token ids as text has them: a token's share falls with its rank."""
    u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
    return (torch.exp(u * math.log(V)) - 1.0).long().clamp_(0, V - 1).to(torch.int32)


def _prepare_embedding(case, g, s):
    N, V, d, ld = case["N"], case["V"], case["d"], case["ld"]
    s["ids"] = _ids(g, N, V)
    s["mask"] = (torch.rand(N, device="cuda", generator=g) >= case["dead"]).to(torch.uint8)
    if case["grad"]:
        s["dout"] = _normal(g, N, d, std=1e-3, type_=case["type"], ld=ld)
        s["dtable"] = torch.empty(V, d, device="cuda")
        # scratch that the trainer keeps: 64 bytes a token, and two fp32 rows for each 32 tokens
        s["ws"] = torch.empty(64 * N + 8 * (d + 64) * (N // 32 + 2) + (1 << 20), dtype=torch.uint8, device="cuda")
    else:
        s["table"] = _normal(g, V, d, std=0.02, type_=case["type"], ld=ld)
        s["out"] = torch.empty(N, d, dtype=TYPES[case["to"]], device="cuda")


def _prepare_residual(case, g, s):
    N, d, ld, t = case["N"], case["d"], case["ld"], case["type"]
    s["x"], s["y"] = _normal(g, N, d, std=2.0, type_=t, ld=ld), _normal(g, N, d, std=0.5, type_=t, ld=ld)
    # a few channels far larger than the rest, as hidden states have them
    hot = torch.randint(0, d, (3,), device="cuda", generator=g)
    s["x"][:, hot] = s["x"][:, hot] * 20.0
    wide = lambda: torch.empty(N, ld, dtype=TYPES[t], device="cuda")[:, :d]  # noqa: E731
    weight = lambda: (1.0 + _normal(g, d, std=0.1)).to(TYPES[case["weight"]])  # noqa: E731
    s["w_pre"], s["w_post"] = weight(), weight() if case["post"] else None
    s["gate"] = {"none": lambda: None, "row": lambda: _normal(g, N, 1), "column": lambda: _normal(g, d, type_=case["weight"]),
                 "full": lambda: _normal(g, N, d, type_=t, ld=ld)}[case["gate"]]()
    s.update(eps=1e-6, residual_scale=1.0, branch_scale=0.7)
    if not case["grad"]:
        s.update(x_out=wide(), h=wide(), rstd_post=torch.empty(N, device="cuda"), rstd_pre=torch.empty(N, device="cuda"))
        return
    # what the forward pass left, and the gradients of its results
    y = s["y"].float()
    s["rstd_post"] = torch.rsqrt(y.square().mean(1) + s["eps"])
    u = y * s["rstd_post"][:, None] * s["w_post"].float() if case["post"] else y
    u = u * s["gate"].float() if s["gate"] is not None else u
    s["x_out"] = wide()
    s["x_out"].copy_(s["x"].float() + 0.7 * u)
    s["rstd_pre"] = torch.rsqrt(s["x_out"].double().square().mean(1) + s["eps"]).float()
    s["dh"], s["dx_out"] = _normal(g, N, d, std=1e-2, type_=t, ld=ld), _normal(g, N, d, std=1e-2, type_=t, ld=ld)
    s.update(dx=wide(), dy=wide(), dw_pre=torch.empty(d, device="cuda"), dw_post=torch.empty(d, device="cuda") if case["post"] else None,
             dgate={"none": lambda: None, "row": lambda: torch.empty(N, 1, device="cuda"),
                    "column": lambda: torch.empty(d, device="cuda"), "full": wide}[case["gate"]](),
             ws=torch.empty(4 * 3 * (d + 64) * 8192 if d < 1024 else 4 * 3 * (d + 64) * 1024, dtype=torch.uint8, device="cuda"))


def _prepare_adjust(case, g, s):
    N, V, per = case["N"], case["V"], case["per"]
    t = TYPES[case["type"]]
    wide = lambda: torch.empty(N, case["ld"], dtype=t, device="cuda")[:, :V]  # noqa: E731
    s["logits"] = _normal(g, N, V, std=3.0, type_=case["type"], ld=case["ld"])
    s["mask"] = None
    if case["penal"]:
        # a request's prompt and what it has answered so far; `per` rows in a row are successive positions of one answer
        requests = -(-N // per)
        prompt = torch.randint(1, case["prompt"] + 1, (requests,), device="cuda", generator=g)
        have = torch.randint(0, case["output"] + 1, (requests,), device="cuda", generator=g)
        width = case["prompt"] + case["output"] + per
        s["tokens"] = _ids(g, requests * width, V)
        row = torch.arange(N, device="cuda")
        begin = (row // per) * width
        first = begin + prompt[row // per]
        last = first + (have[row // per] if per == 1 else (row % per).clamp(max=case["output"]))
        s["spans"] = torch.stack([begin, first, last], 1).contiguous()
        uniform = lambda lo, hi: torch.rand(N, device="cuda", generator=g) * (hi - lo) + lo  # noqa: E731
        s.update(repetition=uniform(1.0, 1.5), frequency=uniform(0.0, 0.5), presence=uniform(-0.5, 0.5))
    if case["bias"]:
        b = case["bias"]
        s["bias_start"] = torch.arange(N + 1, device="cuda") * b
        # different tokens, spread over the vocabulary
        step = max(1, V // b)
        s["bias_id"] = ((torch.arange(N * b, device="cuda") % b) * step
                        + torch.randint(0, step, (N * b,), device="cuda", generator=g)).clamp_(max=V - 1).to(torch.int32)
        s["bias"] = _normal(g, N * b, std=2.0)
    if case["allowed"] < 1.0:
        words = -(-V // 32)
        rare = min(case["allowed"], 1.0 - case["allowed"])
        bits = torch.zeros(N, words, dtype=torch.int32, device="cuda")
        for k in range(32):
            hit = torch.rand(N, words, device="cuda", generator=g) < rare
            bits |= torch.where(hit, torch.tensor(1 << k if k < 31 else -(1 << 31), dtype=torch.int32, device="cuda"), 0)
        s["allowed"] = bits if case["allowed"] < 0.5 else ~bits
    if case["grad"]:
        s["d_out"], s["dlogits"] = _normal(g, N, V, std=1e-2, type_=case["type"], ld=case["ld"]), wide()
    else:
        s["out"] = s["logits"] if case["place"] == "over" else wide()


def _shapes(case):
    """Sizes of the tensors of a case: matrices and vectors of its blocks, then small ones of odd sizes."""
    d, got = case["d"], []
    for _ in range(case["layers"]):
        got += [d * d] * 4 + [4 * d * d] * 3 + [d] * 2
    return got + [1 + 7 * i % 4099 + 13 * (i % 3) for i in range(case["small"])]


def _prepare_clip(case, g, s):
    sizes = _shapes(case)
    s["grads"] = [_normal(g, n, std=1e-3, type_=case["type"]) for n in sizes]
    # the optimizer's one buffer, each tensor on a 16-byte boundary in it
    at, where = 0, []
    for n in sizes:
        where.append(at)
        at += -(-n // 8) * 8
    s["flat"] = torch.zeros(at, dtype=TYPES[case["to"]], device="cuda")
    s["outs"] = [s["flat"][a:a + n] for a, n in zip(where, sizes)]
    s.update(norm=torch.empty(1, device="cuda"), sq_norm=torch.empty(1, device="cuda"), scale=0.25,
             clip=case["ratio"] * 0.25 * 1e-3 * math.sqrt(sum(sizes)), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    if own:
        # the list of tensors, which a trainer makes once: its gradients keep their memory
        from paper_2602_19362_b200 import binding as B
        s["list"] = B.make_tensor_list(s["grads"], s["outs"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    {"embedding": _prepare_embedding, "residual": _prepare_residual, "adjust": _prepare_adjust,
     "clip": _prepare_clip}[case["op"]](case, g, s)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_embedding(s):
    case = s["case"]
    live = s["mask"].bool()[:, None]
    ids = s["ids"].long()
    if not case["grad"]:
        return torch.where(live, s["table"][ids].float() * case["scale"], 0.0).to(TYPES[case["to"]])
    rows = torch.where(live, s["dout"].float() * case["scale"], 0.0)
    return s["dtable"].zero_().index_add_(0, ids, rows)


def _plain_residual(s):
    y, d = s["y"].float(), s["case"]["d"]
    r_post = torch.rsqrt(y.square().mean(1) + s["eps"]) if s["w_post"] is not None else None
    if not s["case"]["grad"]:
        u = y if r_post is None else y * r_post[:, None] * s["w_post"].float()
        u = u if s["gate"] is None else u * s["gate"].float()
        x = s["residual_scale"] * s["x"].float() + s["branch_scale"] * u
        r_pre = torch.rsqrt(x.square().mean(1) + s["eps"])
        out = dict(x_out=x.to(s["x"].dtype), h=(x * r_pre[:, None] * s["w_pre"].float()).to(s["x"].dtype), rstd_pre=r_pre)
        return out if r_post is None else dict(out, rstd_post=r_post)
    t = s["x"].dtype
    x, dh = s["x_out"].float() * s["rstd_pre"][:, None], s["dh"].float()
    wdh = dh * s["w_pre"].float()
    dx_out = s["dx_out"].float() + s["rstd_pre"][:, None] * (wdh - x * (wdh * x).mean(1, keepdim=True))
    out = dict(dx=(s["residual_scale"] * dx_out).to(t), dw_pre=(dh * x).sum(0))
    w = None if s["w_post"] is None else s["w_post"].float()
    n = y if w is None else y * s["rstd_post"][:, None]
    u = n if w is None else n * w
    db = s["branch_scale"] * dx_out
    kind = s["case"]["gate"]
    if kind != "none":
        dgate = db * u
        out["dgate"] = dgate.sum(1, keepdim=True) if kind == "row" else dgate.sum(0) if kind == "column" else dgate.to(t)
        db = db * s["gate"].float()
    if w is not None:
        out["dw_post"] = (db * n).sum(0)
        db = db * w
        db = s["rstd_post"][:, None] * (db - n * (db * n).mean(1, keepdim=True))
    out["dy"] = db.to(t)
    return out


def _seen(s):
    """How often each token is in a row's answer, and whether it is in its prompt or answer."""
    N, V = s["logits"].shape
    case, spans = s["case"], s["spans"]
    longest = case["prompt"] + case["output"]
    at = spans[:, :1] + torch.arange(longest, device=spans.device)
    ids = s["tokens"][at.clamp(max=s["tokens"].numel() - 1)].long()
    hits = torch.zeros(N, V, dtype=torch.int32, device=spans.device)
    count = hits.scatter_add(1, ids, ((at >= spans[:, 1:2]) & (at < spans[:, 2:3])).int())
    return count, hits.scatter_add_(1, ids, (at < spans[:, 2:3]).int()) > 0


def _allowed(s):
    v = torch.arange(s["logits"].shape[1], device="cuda")
    return ((s["allowed"][:, v // 32] >> (v % 32).int()) & 1).bool()


def _plain_adjust(s):
    z = s["logits"].float()
    if s["case"]["grad"]:
        d = s["d_out"].float()
        if "tokens" in s:
            r = s["repetition"][:, None]
            d = torch.where(_seen(s)[1], torch.where(z > 0, d / r, d * r), d)
        if "allowed" in s:
            d = torch.where(_allowed(s), d, 0.0)
        return s["dlogits"].copy_(d)
    if "tokens" in s:
        count, seen = _seen(s)
        r = s["repetition"][:, None]
        z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
        z = z - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if "bias" in s:
        b = s["case"]["bias"]
        z = z.scatter_add(1, s["bias_id"].view(-1, b).long(), s["bias"].view(-1, b))
    if "allowed" in s:
        z = torch.where(_allowed(s), z, -math.inf)
    return s["out"].copy_(z)


def _plain_clip(s):
    sq = torch.stack([(g.float() * s["scale"]).square().sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = sq.sqrt()
    factor = (s["clip"] / (norm + 1e-6)).clamp(max=1.0).float() * s["scale"]
    [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["outs"])]
    return dict(flat=s["flat"], norm=norm.float().view(1), sq_norm=sq.float().view(1))


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"embedding": _plain_embedding, "residual": _plain_residual, "adjust": _plain_adjust, "clip": _plain_clip}[op](s)
    from paper_2602_19362_b200 import binding as B
    if op == "embedding":
        K = B.make_lookup(s["ids"], case["V"], s["mask"], case["scale"])
        if case["grad"]:
            B.oapl_embedding_bwd(K, s["dout"], s["dtable"], False, s["ws"])
            return s["dtable"]
        B.oapl_embedding(K, s["table"], s["out"])
        return s["out"]
    if op == "residual":
        R = B.make_residual(s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["eps"], s["residual_scale"], s["branch_scale"])
        rstd_post = s["rstd_post"] if case["post"] else None
        if case["grad"]:
            B.oapl_residual_norm_bwd(R, s["x_out"], rstd_post, s["rstd_pre"], s["dh"], s["dx_out"], s["dx"], s["dy"], s["dgate"],
                                     s["dw_post"], s["dw_pre"], False, s["ws"])
            keys = ("dx", "dy", "dw_pre") + (("dw_post",) if case["post"] else ()) + (("dgate",) if s["gate"] is not None else ())
        else:
            B.oapl_residual_norm(R, s["x_out"], s["h"], rstd_post, s["rstd_pre"])
            keys = ("x_out", "h", "rstd_pre") + (("rstd_post",) if case["post"] else ())
        return {k: s[k] for k in keys}
    if op == "adjust":
        L = B.make_logits(s["logits"])
        A = B.make_adjust(L, s.get("tokens"), s.get("spans"), s.get("repetition"), s.get("frequency"), s.get("presence"),
                          s.get("bias_start"), s.get("bias_id"), s.get("bias"), s.get("allowed"))
        if case["grad"]:
            B.oapl_logits_adjust_bwd(L, A, s["d_out"], s["dlogits"])
            return s["dlogits"]
        B.oapl_logits_adjust(L, A, s["out"])
        return s["out"]
    B.oapl_grad_norm(s["list"], s["sq_norm"], s["norm"], s["ws"], s["scale"])
    B.oapl_grad_clip(s["list"], s["sq_norm"], s["clip"], s["scale"])
    return dict(flat=s["flat"], norm=s["norm"], sq_norm=s["sq_norm"])


def work(case):
    op = case["op"]
    if op == "embedding":
        N, d, es = case["N"], case["d"], SIZE[case["type"]]
        live = N * (1.0 - case["dead"])
        if case["grad"]:
            return {"bytes": live * d * es + 5 * N + case["V"] * d * 4, "flops": live * d}
        return {"bytes": live * d * es + 5 * N + N * d * SIZE[case["to"]], "flops": live * d}
    if op == "residual":
        N, d, es = case["N"], case["d"], SIZE[case["type"]]
        gate = {"none": 0, "row": 4 * N, "column": d * SIZE[case["weight"]], "full": N * d * es}[case["gate"]]
        if case["grad"]:     # x', y, dh and dx' are read, dx and dy written
            return {"bytes": 6 * N * d * es + 2 * gate + 8 * N + 16 * d, "flops": 25 * N * d}
        return {"bytes": 4 * N * d * es + gate + 8 * N + 8 * d, "flops": 10 * N * d}
    if op == "adjust":
        N, V, es = case["N"], case["V"], SIZE[case["type"]]
        history = (case["prompt"] + case["output"] / 2) if case["penal"] else 0
        history = N * 4 * (history if case["per"] == 1 else history / case["per"])
        bits = N * V / 8 if case["allowed"] < 1.0 else 0
        if case["place"] == "over":     # only what the mask takes is written
            return {"bytes": bits + N * V * es * (1.0 - case["allowed"]) + history, "flops": N * V}
        return {"bytes": bits + 2 * N * V * es + history + 8 * N * case["bias"], "flops": N * V}
    n = sum(_shapes(case))
    # the norm reads all there is before anything can be scaled
    return {"bytes": n * (2 * SIZE[case["type"]] + SIZE[case["to"]]), "flops": 4 * n}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"embedding": _exact_embedding, "residual": _exact_residual, "adjust": _exact_adjust, "clip": _exact_clip}[case["op"]](case, s)


def _exact_embedding(case, s):
    live = s["mask"] != 0
    if not case["grad"]:
        out = torch.zeros(case["N"], case["d"], dtype=torch.float64, device="cuda")
        out[live] = s["table"].index_select(0, s["ids"][live].long()).double() * case["scale"]
        return out
    # sums of sorted rows as differences would cancel: one product per block of columns with a sparse matrix of ones
    at = torch.nonzero(live)[:, 0]
    ids = s["ids"][at].long()
    ones = torch.sparse_coo_tensor(torch.stack([ids, torch.arange(at.numel(), device="cuda")]),
                                   torch.full((at.numel(),), case["scale"], dtype=torch.float64, device="cuda"),
                                   (case["V"], at.numel()))
    return torch.sparse.mm(ones, s["dout"][at].double())


def _exact_residual(case, s):
    """The forward formula in 64 bits; its gradient by automatic differentiation from the stored x'."""
    eps, a, b = s["eps"], s["residual_scale"], s["branch_scale"]
    wide = lambda t: None if t is None else t.double().requires_grad_(case["grad"])  # noqa: E731
    x, y, gate, w_post, w_pre = (wide(s[k]) for k in ("x", "y", "gate", "w_post", "w_pre"))
    norm = lambda v: v / (v.pow(2).sum(1, keepdim=True) / case["d"] + eps).sqrt()  # noqa: E731
    u = norm(y) * w_post if w_post is not None else y
    sum_ = a * x + b * (gate * u if gate is not None else u)
    if not case["grad"]:
        rstd = lambda v: 1.0 / ((v * v).sum(1) / case["d"] + eps).sqrt()  # noqa: E731
        out = dict(x_out=sum_, h=norm(sum_) * w_pre, rstd_pre=rstd(sum_))
        return dict(out, rstd_post=rstd(y)) if w_post is not None else out
    stored = wide(s["x_out"])
    d_stored, dw_pre = torch.autograd.grad(norm(stored) * w_pre, [stored, w_pre], s["dh"].double())
    leaves = dict(dx=x, dy=y, dgate=gate, dw_post=w_post)
    leaves = {k: v for k, v in leaves.items() if v is not None}
    got = torch.autograd.grad(sum_, list(leaves.values()), d_stored + s["dx_out"].double())
    return dict(zip(leaves, got), dw_pre=dw_pre)


def _exact_adjust(case, s):
    out = torch.empty(case["N"], case["V"], dtype=torch.float64, device="cuda")
    for n in range(case["N"]):
        z = s["logits"][n].double()
        d = s["d_out"][n].double() if case["grad"] else None
        if case["penal"]:
            lo, mid, hi = s["host_spans"][n] if "host_spans" in s else s.setdefault("host_spans", s["spans"].tolist())[n]
            r, f, p = (s[k][n].double() for k in ("repetition", "frequency", "presence"))
            answer = torch.bincount(s["tokens"][mid:hi].long(), minlength=case["V"])
            seen = torch.bincount(s["tokens"][lo:hi].long(), minlength=case["V"]) != 0
            slope = torch.where(seen, torch.where(z > 0, 1.0 / r, r), torch.ones_like(z))
            z = z * slope - f * answer - p * (answer != 0)
            d = d * slope if d is not None else None
        if case["bias"]:
            of = slice(n * case["bias"], (n + 1) * case["bias"])
            z = z.index_add(0, s["bias_id"][of].long(), s["bias"][of].double())
        if case["allowed"] < 1.0:
            word = s["allowed"][n].long()[:, None]
            closed = (torch.bitwise_right_shift(word, torch.arange(32, device="cuda")) & 1).reshape(-1)[:case["V"]] == 0
            z[closed] = -math.inf
            if d is not None:
                d[closed] = 0.0
        out[n] = z if d is None else d
    return out


def _exact_clip(case, s):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"])) * s["scale"]
    factor = min(1.0, s["clip"] / (norm + 1e-6)) * s["scale"]
    flat = torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda")
    at = 0
    for g in s["grads"]:
        flat[at:at + g.numel()] = g.double() * factor
        at += -(-g.numel() // 8) * 8
    return dict(flat=flat, norm=torch.tensor([norm], dtype=torch.float64), sq_norm=torch.tensor([norm * norm], dtype=torch.float64))
