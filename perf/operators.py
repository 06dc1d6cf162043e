"""Cases for the operators around the LM head: log-probabilities of given tokens with entropy and top
alternatives from logits in memory, their gradient, quantisation to 8-bit floating point with a scale per
block of 128, and the matrix product of two matrices held that way.

Each case is a dict with an "op":
  logprobs   rows of logits -> log-probability of the row's token, entropy, log-sum-exp, top alternatives
  gradient   gradients of those outputs -> gradient of the logits
  quantize   a matrix -> 8-bit values and one scale per 1 x 128 or 128 x 128 block
  matmul     C = A . B^T of two such matrices

`own` selects what `run` computes with: elementary torch operations in fp32, or the library's entry points.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
         "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
SMALLEST_AMAX = 2.0 ** -100     # a block's largest magnitude is taken to be at least this


def listed():
    return [
        # one decoded token: the engine reports its log-probability and twenty alternatives
        dict(name="logprobs one token", op="logprobs", N=1, V=152064, ld=152064, type="bf16", K=20, dead=0.0),
        # a decode batch whose engine hands over fp32 logits
        dict(name="logprobs decode batch", op="logprobs", N=64, V=128256, ld=128256, type="f32", K=5, dead=0.0),
        # a row chunk of a trainer that re-scores responses, with the entropy it logs
        dict(name="logprobs trainer chunk", op="logprobs", N=4096, V=152064, ld=152064, type="bf16", K=8, dead=0.0),
        # an odd vocabulary in rows that are no multiple of 16 bytes, a third of the rows padding
        dict(name="logprobs ragged", op="logprobs", N=1531, V=50021, ld=50023, type="f16", K=3, dead=0.33),
        # the trainer chunk's backward pass
        dict(name="gradient trainer chunk", op="gradient", N=4096, V=152064, ld=152064, type="bf16", K=0, dead=0.0),
        # distillation on a teacher's eight alternatives, fp32 logits, some padding
        dict(name="gradient distillation", op="gradient", N=257, V=32003, ld=32003, type="f32", K=8, dead=0.2),
        # hidden states on their way into an 8-bit product
        dict(name="quantize rows", op="quantize", R=8192, C=3584, ld=3584, type="bf16", to="e4m3", block=1, turn=False),
        # the LM-head weight, once per optimizer step
        dict(name="quantize weight", op="quantize", R=152064, C=3584, ld=3584, type="bf16", to="e4m3", block=128,
             turn=False),
        # a chunk of logit gradients, turned so that its rows become the contracted axis of dW
        dict(name="quantize turned", op="quantize", R=1999, C=50021, ld=50024, type="bf16", to="e5m2", block=1, turn=True),
        # the logits of a row chunk
        dict(name="matmul logits", op="matmul", M=4096, N=152064, K=3584, a="e4m3", b="e4m3", block=128, out="bf16"),
        # the logits of four decoded tokens
        dict(name="matmul decode", op="matmul", M=4, N=152064, K=3584, a="e4m3", b="e4m3", block=128, out="bf16"),
        # the weight gradient of a chunk: a scale per row and 128 tokens on both sides, fp32 result
        dict(name="matmul weight gradient", op="matmul", M=50021, N=1536, K=1999, a="e5m2", b="e4m3", block=1,
             out="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "gradient", "quantize", "matmul"])
    if op in ("logprobs", "gradient"):
        type_ = rng.choice(["bf16", "bf16", "f16", "f32"])
        V = _log_int(rng, 1000, 152064)
        N = _log_int(rng, 1, min(16384, (4096 * 152064 if type_ != "f32" else 2048 * 152064) // (V + 64)))
        ld = V + rng.choice([0, 0, (-V) % 8, rng.randint(1, 64)])
        return dict(op=op, N=N, V=V, ld=ld, type=type_, K=rng.choice([0, 1, 5, 20, 32]), dead=rng.choice([0.0, 0.0, 0.3]))
    if op == "quantize":
        turn = rng.random() < 0.4
        C = _log_int(rng, 64, 60000)
        R = _log_int(rng, 1, min(152064, 152064 * 3584 // C))
        return dict(op=op, R=R, C=C, ld=C + rng.choice([0, (-C) % 8, rng.randint(1, 20)]), type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    to=rng.choice(["e4m3", "e4m3", "e5m2"]), block=rng.choice([1, 128]), turn=turn)
    M = _log_int(rng, 1, 8192)
    N = _log_int(rng, 200, 152064)
    K = _log_int(rng, 64, min(20000, 4096 * 152064 * 3584 // (M * N)))
    return dict(op="matmul", M=M, N=N, K=K, a=rng.choice(["e4m3", "e4m3", "e5m2"]), b="e4m3", block=rng.choice([128, 128, 1]),
                out=rng.choice(["bf16", "bf16", "f16", "f32"]))


# ------------------------------------------------------------------------------------------------ inputs

def _logits(case, g):
    """Rows of logits as an LM head gives them: a bell of about two, and a few tokens far above it."""
    N, V = case["N"], case["V"]
    buf = torch.empty(N, case["ld"], dtype=TYPES[case["type"]], device="cuda").normal_(0.0, 2.0, generator=g)
    z = buf[:, :V]
    at = torch.randint(0, V, (N, 6), device="cuda", generator=g)
    up = torch.rand(N, 6, device="cuda", generator=g) * 14.0
    z.scatter_(1, at, (z.gather(1, at).float() + up).to(z.dtype))
    # four tokens of five are one of those that the row favours
    pick = torch.rand(N, device="cuda", generator=g) < 0.8
    targets = torch.where(pick, at[:, 0], torch.randint(0, V, (N,), device="cuda", generator=g)).to(torch.int32)
    mask = (torch.rand(N, device="cuda", generator=g) >= case["dead"]).to(torch.uint8)
    return z, targets, mask


def _scaled(rows, K, kind, block, g):
    """A quantised matrix: values that fill the type's range as a block's largest magnitude makes them, and its scales."""
    ld = -(-K // 16) * 16
    kb = -(-K // 128)
    top = LARGEST[kind]
    data = torch.empty(rows, ld, dtype=torch.float32, device="cuda").normal_(0.0, top / 3.5, generator=g)
    data = data.clamp_(-top, top).to(TYPES[kind])[:, :K]
    scale = torch.empty(kb, -(-rows // block), dtype=torch.float32, device="cuda").uniform_(0.5, 2.0, generator=g)
    return dict(data=data, scale=(scale * (3.5 / top / 8.0)).t(), block=block)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(case=case)
    if op in ("logprobs", "gradient"):
        N, K = case["N"], case["K"]
        z, targets, mask = _logits(case, g)
        s.update(logits=z, targets=targets, mask=mask)
        if op == "logprobs":
            s.update(token_logp=torch.empty(N, device="cuda"), token_entropy=torch.empty(N, device="cuda"),
                     token_lse=torch.empty(N, device="cuda"),
                     top_logp=torch.empty(N, K, device="cuda") if K else None,
                     top_id=torch.empty(N, K, dtype=torch.int32, device="cuda") if K else None)
        else:
            # what the forward pass left, and the gradients of its outputs
            x = z.float()
            lse = torch.logsumexp(x, 1)
            ent = lse - (torch.softmax(x, 1) * x).sum(1)
            live = mask.bool()
            ids = torch.topk(x, K, 1).indices.to(torch.int32) if K else None
            del x
            s.update(token_lse=torch.where(live, lse, 0.0), token_entropy=torch.where(live, ent, 0.0),
                     g_logp=torch.randn(N, device="cuda", generator=g), g_entropy=0.1 * torch.randn(N, device="cuda", generator=g),
                     g_top=torch.rand(N, K, device="cuda", generator=g) if K else None, top_id=ids,
                     dlogits=torch.empty(N, case["ld"], dtype=z.dtype, device="cuda")[:, :case["V"]])
    elif op == "quantize":
        R, C = case["R"], case["C"]
        buf = torch.empty(R, case["ld"], dtype=TYPES[case["type"]], device="cuda").normal_(0.0, 1.0, generator=g)
        x = buf[:, :C]
        # a few columns far larger than the rest, as hidden states have them
        hot = torch.randint(0, C, (4,), device="cuda", generator=g)
        x[:, hot] = x[:, hot] * 30.0
        rows, cols = (C, R) if case["turn"] else (R, C)
        b = case["block"]
        s.update(x=x, q=torch.empty(rows, -(-cols // 16) * 16, dtype=TYPES[case["to"]], device="cuda")[:, :cols],
                 scale=torch.empty(-(-cols // 128), -(-rows // b), device="cuda").t())
    else:
        s.update(a=_scaled(case["M"], case["K"], case["a"], 1, g), b=_scaled(case["N"], case["K"], case["b"], case["block"], g),
                 c=torch.empty(case["M"], case["N"], dtype=TYPES[case["out"]], device="cuda"))
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_logprobs(s):
    K = s["case"]["K"]
    live = s["mask"].bool()
    z = s["logits"].float() + 0.0
    V = z.shape[1]
    m = z.max(1, keepdim=True).values
    d = z - m
    e = torch.exp(d)
    total = e.sum(1)
    log_total = torch.log(total)
    entropy = log_total - (e * d).sum(1) / total
    del d, e
    lse = m[:, 0] + log_total
    logp = z.gather(1, s["targets"].long()[:, None])[:, 0] - lse
    out = dict(token_logp=torch.where(live, logp, 0.0), token_entropy=torch.where(live, entropy, 0.0),
               token_lse=torch.where(live, lse, 0.0))
    if K:
        # one whole number per entry that orders by value, then by the lower index
        bits = z.view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
        key += (V - 1) - torch.arange(V, device=z.device)
        best = torch.topk(key, min(K, V), 1, sorted=True).values
        ids = (V - 1) - (best & 0xFFFFFFFF)
        out["top_logp"] = torch.where(live[:, None], z.gather(1, ids) - lse[:, None], 0.0)
        out["top_id"] = torch.where(live[:, None], ids, -1).to(torch.int32)
    return out


def _plain_gradient(s):
    K = s["case"]["K"]
    live = s["mask"].bool()[:, None]
    lp = s["logits"].float() - s["token_lse"][:, None]
    p = torch.exp(lp)
    weight = s["g_logp"] + s["g_top"].sum(1) if K else s["g_logp"]
    d = -p * (weight[:, None] + s["g_entropy"][:, None] * (lp + s["token_entropy"][:, None]))
    d.scatter_add_(1, s["targets"].long()[:, None], s["g_logp"][:, None])
    if K:
        d.scatter_add_(1, s["top_id"].long(), s["g_top"])
    return torch.where(live, d, 0.0).to(s["logits"].dtype)


def _blocks(x, block, cols=128):
    """x, padded with zeros, as [row blocks, block, column blocks, cols]."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, (-c) % cols, 0, (-r) % block))
    return x.view(x.shape[0] // block, block, x.shape[1] // cols, cols)


def _plain_quantize(s):
    case = s["case"]
    x = s["x"].float()
    if case["turn"]:
        x = x.t()
    rows, cols = x.shape
    blocks = _blocks(x, case["block"])
    amax = blocks.abs().amax((1, 3)).clamp_min(SMALLEST_AMAX)
    top = LARGEST[case["to"]]
    scale = amax / top
    # x * top / amax, with top = 0.875 * 2^e: both factors of 16-bit inputs are exact, so ties stay ties
    q = (blocks * 0.875) / (amax * (0.875 / top))[:, None, :, None]
    q = q.flatten(2).flatten(0, 1)[:rows, :cols]
    return dict(q=q.clamp(-top, top).to(TYPES[case["to"]]), scale=scale)


def _widen(m, dtype):
    """The matrix that data and scales stand for."""
    x = m["data"].to(dtype)
    rows, cols = x.shape
    s = m["scale"].to(dtype)
    x = _blocks(x, m["block"]) * s[:, None, :, None]
    return x.flatten(2).flatten(0, 1)[:rows, :cols]


def _plain_matmul(s):
    a, b = _widen(s["a"], torch.float32), _widen(s["b"], torch.float32)
    return (a @ b.t()).to(s["c"].dtype)


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2602_19362_b200 import binding as B
        if op == "logprobs":
            L = B.make_logits(s["logits"], s["targets"], s["mask"])
            B.oapl_logits_logprobs(L, s["token_logp"], s["token_entropy"], s["token_lse"], s["top_logp"], s["top_id"])
            keys = ("token_logp", "token_entropy", "token_lse") + (("top_logp", "top_id") if s["top_id"] is not None else ())
            return {k: s[k] for k in keys}
        if op == "gradient":
            L = B.make_logits(s["logits"], s["targets"], s["mask"])
            B.oapl_logits_logprobs_bwd(L, s["token_lse"], s["token_entropy"], s["g_logp"], s["g_entropy"], s["g_top"],
                                       s["top_id"], s["dlogits"])
            return s["dlogits"]
        if op == "quantize":
            Q = B.make_scaled(s["q"], s["scale"], s["case"]["block"])
            B.oapl_quantize(s["x"], Q, transpose=s["case"]["turn"])
            return dict(q=s["q"], scale=s["scale"])
        A = B.make_scaled(s["a"]["data"], s["a"]["scale"], s["a"]["block"])
        W = B.make_scaled(s["b"]["data"], s["b"]["scale"], s["b"]["block"])
        B.oapl_scaled_matmul(A, W, s["c"])
        return s["c"]
    if op == "logprobs":
        return _plain_logprobs(s)
    if op == "gradient":
        return _plain_gradient(s)
    if op == "quantize":
        return _plain_quantize(s)
    return _plain_matmul(s)


def work(case):
    op = case["op"]
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if op in ("logprobs", "gradient"):
        # masked rows are not read; the gradient of a masked row is still written
        N, V, K = case["N"], case["V"], case["K"]
        live = N * (1.0 - case["dead"])
        entries = live * V
        if op == "logprobs":
            return {"bytes": entries * size[case["type"]] + N * (12 + 8 * K + 5), "flops": 5 * entries}
        return {"bytes": (entries + N * V) * size[case["type"]] + N * (16 + 8 * K + 5), "flops": 6 * entries}
    if op == "quantize":
        R, C, b = case["R"], case["C"], case["block"]
        rows, cols = (C, R) if case["turn"] else (R, C)
        return {"bytes": R * C * (size[case["type"]] + 1) + 4 * -(-rows // b) * -(-cols // 128), "flops": 3 * R * C}
    M, N, K, b = case["M"], case["N"], case["K"], case["block"]
    kb = -(-K // 128)
    return {"bytes": (M + N) * K + 4 * kb * (M + -(-N // b)) + M * N * size[case["out"]], "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "logprobs":
        K, V = case["K"], case["V"]
        parts = []
        for r in range(0, case["N"], 256):
            z = s["logits"][r:r + 256].double()
            ln_p = torch.log_softmax(z, 1)
            live = s["mask"][r:r + 256].bool()
            one = dict(token_logp=ln_p.gather(1, s["targets"][r:r + 256].long()[:, None])[:, 0] * live,
                       token_entropy=-(ln_p.exp() * ln_p).sum(1) * live, token_lse=torch.logsumexp(z, 1) * live)
            if K:
                best = torch.sort(ln_p, dim=1, descending=True, stable=True)
                one["top_logp"] = best.values[:, :K] * live[:, None]
                # several values of z can share one ln_p in 64 bits only where they are equal
                one["top_id"] = torch.where(live[:, None], best.indices[:, :K], -1).to(torch.int32)
            parts.append(one)
        return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if op == "gradient":
        out = torch.zeros(case["N"], case["V"], dtype=torch.float64, device="cuda")
        for r in range(0, case["N"], 256):
            w = slice(r, r + 256)
            p = torch.exp(s["logits"][w].double() - s["token_lse"][w].double()[:, None])
            ln_p = s["logits"][w].double() - s["token_lse"][w].double()[:, None]
            gl, ge, h = (s[k][w].double()[:, None] for k in ("g_logp", "g_entropy", "token_entropy"))
            hot = torch.zeros_like(p).scatter_(1, s["targets"][w].long()[:, None], 1.0)
            d = gl * (hot - p) - ge * p * (ln_p + h)
            for k in range(case["K"]):
                gk = s["g_top"][w, k].double()[:, None]
                d += gk * (torch.zeros_like(p).scatter_(1, s["top_id"][w, k].long()[:, None], 1.0) - p)
            out[w] = d * s["mask"][w].bool()[:, None]
        return out
    if op == "quantize":
        x = s["x"].t() if case["turn"] else s["x"]
        rows, cols = x.shape
        b, top = case["block"], LARGEST[case["to"]]
        amax = torch.zeros(-(-rows // b), -(-cols // 128), dtype=torch.float64, device="cuda")
        values = torch.empty(rows, cols, dtype=TYPES[case["to"]], device="cuda")
        for j in range(0, cols, 128):
            part = x[:, j:j + 128].double()
            one = torch.nn.functional.pad(part.abs().amax(1), (0, (-rows) % b)).view(-1, b).amax(1).clamp_min(SMALLEST_AMAX)
            amax[:, j // 128] = one
            # rounding to 32 bits on the way is far finer than the step of the 8-bit type
            values[:, j:j + 128] = (part * top / one.repeat_interleave(b)[:rows, None]).float().to(values.dtype)
        return dict(q=values, scale=amax / top)
    return _widen64(s["a"]) @ _widen64(s["b"]).t()


def _widen64(m):
    x = m["data"].double()
    by_row = m["scale"].double().repeat_interleave(m["block"], 0)[:x.shape[0]]
    return x * by_row.repeat_interleave(128, 1)[:, :x.shape[1]]
