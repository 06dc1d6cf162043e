"""A trainer step with tied weights through all of its operators: embedding, residual norm, the loss on the LM head and
its gradient, back through the norm into the embedding, whose gradient is added to the head's; the gradient norm over
all parameters and the optimizer step.  Against the 64-bit oracle of the head and automatic differentiation."""
import dataclasses
import math

import numpy as np
import pytest
import torch

from oracle import oapl_oracle as orc
from paper_2602_19362_b200 import binding as B, synth
from tests import helpers as hp

pytestmark = pytest.mark.gpu


def _batch(seed):
    wl = dataclasses.replace(synth.small_variant("14b-long", prompts=4, samples=3, live_rows=300), d=128, V=512)
    cpu = synth.make_batch(wl, seed=seed)
    return cpu, hp.to_dev(cpu)


class Step:
    """Everything that a trainer keeps: weights, buffers, workspaces."""

    def __init__(self, dev, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        N, d, V, S, P = (dev[k] for k in "NdVSP")
        bf = lambda *s: torch.randn(*s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
        self.dev, self.N, self.d, self.V = dev, N, d, V
        self.W = (bf(V, d).float() / math.sqrt(d)).to(torch.bfloat16)
        self.ids = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
        self.y, self.gate = bf(N, d), bf(d)
        self.w_post, self.w_pre = (1 + 0.1 * bf(d).float()).to(torch.bfloat16), (1 + 0.1 * bf(d).float()).to(torch.bfloat16)
        new = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.x, self.H, self.dH, self.dx, self.dy = (new(N, d) for _ in range(5))
        self.rp, self.rq = new(N, t=f32), new(N, t=f32)
        self.dW, self.dw_post, self.dw_pre, self.dgate = new(V, d, t=f32), new(d, t=f32), new(d, t=f32), new(d, t=f32)
        self.loss, self.seq_logp, self.vhat, self.delta, self.tok = (new(n, t=f32) for n in (1, S, P, S, N))
        self.sq, self.norm = new(1, t=f32), new(1, t=f32)
        self.scale = 3.0
        self.lookup = B.make_lookup(self.ids, V, None, self.scale)
        self.res = B.make_residual(self.x, self.y, self.gate, self.w_post, self.w_pre, 1e-6, 1.0, 0.5)
        self.prob = B.make_problem({**dev, "H": self.H, "W": self.W})
        self.ws = B.alloc_workspace(self.prob, B.OAPL_FLAG_FUSED)
        u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.ws_e = u8(B.oapl_embedding_workspace_bytes(N, V, d))
        self.ws_r = u8(B.oapl_residual_norm_workspace_bytes(N, d))
        # the head's own gradient goes to the optimizer step by itself: it adds its squares to these
        self.rest = B.make_tensor_list([self.dw_post, self.dw_pre, self.dgate])
        self.ws_n = u8(B.oapl_grad_norm_workspace_bytes(3))
        self.x0 = new(N, d)
        self.xo = new(N, d)

    def run(self):
        B.oapl_embedding(self.lookup, self.W, self.x)
        B.oapl_residual_norm(self.res, self.xo, self.H, self.rp, self.rq)
        B.oapl_loss_fwd_bwd(self.prob, self.loss, self.seq_logp, self.vhat, self.delta, self.tok, self.dH, self.dW, False, self.ws)
        B.oapl_residual_norm_bwd(self.res, self.xo, self.rp, self.rq, self.dH, None, self.dx, self.dy, self.dgate, self.dw_post,
                                 self.dw_pre, False, self.ws_r)
        B.oapl_embedding_bwd(self.lookup, self.dx, self.dW, True, self.ws_e)
        B.oapl_grad_norm(self.rest, self.sq, self.norm, self.ws_n)


def _reference(s, cpu):
    """The step in 64 bits from the same bf16 weights; nothing in between is rounded."""
    leaves = {k: getattr(s, k).double().requires_grad_() for k in ("W", "y", "gate", "w_post", "w_pre")}
    n = lambda m: m / (m.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    x = leaves["W"][s.ids.long()] * s.scale
    H = n(x + 0.5 * leaves["gate"] * n(leaves["y"]) * leaves["w_post"]) * leaves["w_pre"]
    Hn, Wn = H.detach().cpu().numpy(), s.W.double().cpu().numpy()
    ref = orc.loss_fwd(Hn, Wn, hp.npy(cpu["targets"]), hp.npy(cpu["mask"]), hp.npy(cpu["seq_id"]), hp.npy(cpu["group_id"]),
                       hp.npy(cpu["reward"]), hp.npy(cpu["logp_inf"]), cpu["S"], cpu["P"], cpu["beta_v"], cpu["beta_loss"],
                       cpu["loss_scale"])
    dH, dW = orc.loss_bwd(Hn, Wn, hp.npy(cpu["targets"]), hp.npy(cpu["mask"]), hp.npy(cpu["seq_id"]), ref["coef"])
    grads = dict(zip(leaves, torch.autograd.grad(H, list(leaves.values()), torch.from_numpy(dH).cuda())))
    grads["W"] = grads["W"] + torch.from_numpy(dW).cuda()
    return ref, {k: v.cpu().numpy() for k, v in grads.items()}


def test_step_with_tied_weights():
    cpu, dev = _batch(3)
    s = Step(dev, 4)
    s.run()
    assert B.oapl_get_last_status(s.ws) == 0
    ref, grads = _reference(s, cpu)
    # H is rounded to bf16 before the logits, so a log-probability moves by up to 2^-9 |H| |W| per term: the path's
    # tolerances are those of its own tests, twice as wide for what passes a second rounding (x', H, dH, dx)
    assert abs(float(s.loss) - ref["loss"]) <= 1e-2 * abs(ref["loss"])
    for k, got in (("W", s.dW), ("gate", s.dgate), ("w_post", s.dw_post), ("w_pre", s.dw_pre), ("y", s.dy)):
        assert hp.fro_rel(hp.f64(got), grads[k]) <= 2 * hp.TOL_FRO, k
    rest = math.sqrt(sum(float(t.double().square().sum()) for t in (s.dw_post, s.dw_pre, s.dgate)))
    assert float(s.norm) == pytest.approx(rest, rel=1e-6)
    # the optimizer clips by the norm over the head and the rest
    m, v, master, gn = torch.zeros_like(s.dW), torch.zeros_like(s.dW), s.W.float(), torch.zeros(1, device="cuda")
    B.oapl_adamw_step(s.W, master, s.dW.view(-1), m, v, 1, 1e-3, 0.9, 0.95, 1e-8, 0.0, 0.1, s.sq, gn)
    whole = math.sqrt(rest ** 2 + float(s.dW.double().square().sum()))
    assert float(gn) == pytest.approx(whole, rel=1e-5)
    assert hp.fro_rel(hp.f64(m), 0.1 * hp.f64(s.dW) * min(1.0, 0.1 / whole)) <= 1e-5


def test_step_captured_and_replayed_with_new_weights():
    cpu, dev = _batch(5)
    s = Step(dev, 6)
    s.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s.run()
    torch.cuda.synchronize()
    for k in range(2):
        s.W.mul_(1.25)
        s.y.mul_(0.5)
        s.run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (s.loss, s.H, s.dW, s.dy, s.dgate, s.dw_post, s.dw_pre, s.norm)]
        for t in (s.H, s.dW, s.dy, s.dgate):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = (s.loss, s.H, s.dW, s.dy, s.dgate, s.dw_post, s.dw_pre, s.norm)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), k
    graph.reset()
    assert np.isfinite(float(s.loss))
