"""Refusals of the embedding, the residual norm, the gradient norm and clipping, and the adjustments of logits: all are
made on the host, before any CUDA call, so they are tested without a GPU (the addresses are never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2602_19362_b200 import binding as B, build

ST = ctypes.c_void_p(0)
INVALID, MISALIGNED, SMALL, UNSUPPORTED = -1, -2, -3, -4
NAN, INF = float("nan"), float("inf")
GB = 1 << 30


def at(gb, off=0):
    """Addresses a few gigabytes apart, so that nothing overlaps by chance."""
    return gb * 64 * GB + off


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def _set(s, kw):
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _lookup(**kw):
    return _set(B.OaplLookup(at(1), at(2), 64, 1000, 1.0), kw)


@pytest.mark.parametrize("kw, want", [
    (dict(ids=0), INVALID), (dict(N=0), INVALID), (dict(N=-1), INVALID), (dict(V=0), INVALID), (dict(scale=NAN), INVALID),
    (dict(scale=INF), INVALID), (dict(ids=at(1, 2)), MISALIGNED), (dict(N=3 * 10 ** 9), UNSUPPORTED),
    (dict(V=2 * 10 ** 9 + 1), UNSUPPORTED)])
def test_lookup_struct(L, kw, want):
    k = _lookup(**kw)
    assert L.oapl_embedding(k, at(3), 0, 128, 128, at(4), 0, 128, None, ST) == want
    assert L.oapl_embedding_bwd(k, at(3), 0, 128, 128, at(4), 128, 0, None, at(5), 1 << 50, ST) == want


def test_embedding_arguments(L):
    def f(table=at(3), tt=0, ld=128, d=128, out=at(4), ot=0, ldo=128, k=_lookup()):
        return L.oapl_embedding(k, table, tt, ld, d, out, ot, ldo, None, ST)
    assert f(k=None) == f(table=None) == f(out=None) == f(tt=3) == f(ot=-1) == f(ld=127) == f(ldo=127) == f(d=0) == INVALID
    assert f(table=at(3, 1)) == f(out=at(4, 1)) == f(tt=2, table=at(3, 2)) == MISALIGNED
    # the result over the table, or into its rows
    assert f(out=at(3)) == f(out=at(3, 999 * 256)) == INVALID


def test_embedding_gradient_arguments(L):
    def f(dout=at(3), t=0, ld=128, d=128, dt=at(4), ldt=128, ws=at(5), n=1 << 50, k=_lookup()):
        return L.oapl_embedding_bwd(k, dout, t, ld, d, dt, ldt, 0, None, ws, n, ST)
    assert f(k=None) == f(dout=None) == f(dt=None) == f(ws=None) == f(t=4) == f(ld=127) == f(ldt=100) == f(d=-1) == INVALID
    assert f(dout=at(3, 1)) == f(dt=at(4, 2)) == f(ws=at(5, 8)) == MISALIGNED
    assert f(dt=at(3, 256)) == INVALID
    need = L.oapl_embedding_workspace_bytes(64, 1000, 128)
    assert need > 0 and f(n=need - 1) == SMALL


def test_embedding_workspace(L):
    w = L.oapl_embedding_workspace_bytes
    assert w(0, 10, 10) == w(10, 0, 10) == w(10, 10, 0) == w(3 * 10 ** 9, 10, 10) == 0
    # two rows of partial sums and a word for each chunk, the list, and for many rows a second list and the digits' counts
    assert w(1, 10, 64) <= 256 + 512 + 256
    for N, chunk in ((8192, 32), (40960, 32), (300000, 128), (4000000, 256)):
        assert w(N, 152064, 64) <= 16 * N + 516 * (N // chunk + 1) + 4 * 1024 * (N // 2048 + 2) + 2048


def _residual(**kw):
    r = B.OaplResidual(64, 128, 0, at(1), 128, at(2), 128, None, 0, 0, 0, at(3), at(4), 0, 0.0, 1e-6, 1.0, 1.0)
    return _set(r, kw)


def _fwd(L, r, x_out=at(10), ldx=128, h=at(11), ldh=128, rp=at(12), rq=at(13)):
    return L.oapl_residual_norm(r, x_out, ldx, h, ldh, rp, rq, ST)


def _bwd(L, r, **kw):
    a = dict(x_out=at(10), ldxo=128, rp=at(12), rq=at(13), dh=at(14), lddh=128, dxo=at(15), lddxo=128, dx=at(16), lddx=128,
             dy=at(17), lddy=128, dg=None, lddg=0, dwp=at(19), dwq=at(20), acc=0, ws=at(21), n=1 << 50)
    a.update(kw)
    return L.oapl_residual_norm_bwd(r, *a.values(), ST)


@pytest.mark.parametrize("kw, want", [
    (dict(N=0), INVALID), (dict(N=-5), INVALID), (dict(d=0), INVALID), (dict(type=3), INVALID), (dict(ld_x=127), INVALID),
    (dict(ld_y=127), INVALID), (dict(y=0), INVALID), (dict(gate_kind=2), INVALID), (dict(gate=at(5)), INVALID),
    (dict(gate_kind=4, gate=at(5)), INVALID), (dict(gate_kind=2, gate=at(5), gate_type=3), INVALID),
    (dict(gate_kind=3, gate=at(5), ld_gate=127), INVALID), (dict(gate_kind=3, gate=at(5), ld_gate=128, gate_type=2), INVALID),
    (dict(gate_kind=1, gate=at(5), ld_gate=0), INVALID), (dict(weight_type=5), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(weight_offset=NAN), INVALID), (dict(residual_scale=INF), INVALID),
    (dict(branch_scale=NAN), INVALID), (dict(x=at(1, 1)), MISALIGNED), (dict(y=at(2, 1)), MISALIGNED),
    (dict(gate_kind=2, gate=at(5, 2), gate_type=2), MISALIGNED), (dict(w_post=at(3, 1)), MISALIGNED),
    (dict(w_pre=at(4, 2), weight_type=2), MISALIGNED), (dict(N=3 * 10 ** 9), UNSUPPORTED),
    (dict(d=16385, ld_x=20000, ld_y=20000), UNSUPPORTED)])
def test_residual_struct(L, kw, want):
    r = _residual(**kw)
    assert _fwd(L, r, ldx=1 << 20, ldh=1 << 20) == want
    assert _bwd(L, r, ldxo=1 << 20, lddh=1 << 20, lddxo=1 << 20, lddx=1 << 20, lddy=1 << 20) == want


def test_residual_arguments(L):
    r = _residual()
    assert _fwd(L, None) == INVALID
    assert _fwd(L, _residual(x=0)) == INVALID
    assert _fwd(L, r, h=None) == INVALID                                   # a weight without a place for its result
    assert _fwd(L, _residual(w_pre=0)) == INVALID                          # and the other way round
    assert _fwd(L, _residual(w_pre=0), x_out=None, h=None, rq=None) == INVALID
    assert _fwd(L, _residual(w_post=0)) == INVALID                         # statistics of a norm that is not there
    assert _fwd(L, _residual(y=0, w_post=0, w_pre=0), h=None, rp=None, rq=None) == INVALID
    assert _fwd(L, r, ldx=127) == _fwd(L, r, ldh=1) == INVALID
    assert _fwd(L, r, x_out=at(10, 1)) == _fwd(L, r, h=at(11, 1)) == _fwd(L, r, rp=at(12, 2)) == MISALIGNED
    # over an input only row by row, and never over one another
    assert _fwd(L, r, x_out=at(1, 256)) == _fwd(L, r, h=at(2, 2)) == _fwd(L, r, h=at(1), ldh=136) == INVALID
    assert _fwd(L, r, h=at(10)) == _fwd(L, r, h=at(10, 256 * 63)) == INVALID


def test_residual_gradient_arguments(L):
    r = _residual()
    f = lambda **kw: _bwd(L, kw.pop("r", r), **kw)  # noqa: E731
    assert f(r=None) == f(x_out=None) == f(rp=None) == f(rq=None) == f(dh=None) == INVALID
    assert f(r=_residual(w_pre=0)) == INVALID                              # dh without its norm
    assert f(r=_residual(w_pre=0), dh=None, dwq=None, dxo=None) == INVALID  # no gradient at all
    assert f(r=_residual(w_post=0)) == INVALID
    assert f(r=_residual(y=0, w_post=0), dwp=None) == INVALID              # dy without y
    assert f(dg=at(18), lddg=1) == INVALID                                 # dgate without a gate
    assert f(dx=None, dy=None, dwp=None, dwq=None) == INVALID
    assert f(ldxo=127) == f(lddh=127) == f(lddxo=127) == f(lddx=127) == f(lddy=127) == INVALID
    full = _residual(gate_kind=3, gate=at(5), ld_gate=128)
    assert f(r=full, dg=at(18), lddg=127) == INVALID
    assert f(dx=at(16, 1)) == f(dh=at(14, 1)) == f(dwp=at(19, 2)) == f(ws=at(21, 8)) == MISALIGNED
    assert f(ws=None) == INVALID
    need = L.oapl_residual_norm_workspace_bytes(64, 128)
    assert need >= 3 * 4 * 128 * 64 and f(n=need - 1) == SMALL
    assert f(dy=at(16)) == f(dx=at(14, 256)) == f(dy=at(2), lddy=136) == INVALID
    assert f(r=full, dg=at(17), lddg=128) == INVALID
    assert L.oapl_residual_norm_workspace_bytes(0, 128) == L.oapl_residual_norm_workspace_bytes(5, 16385) == 0


def _tensors(*kw):
    return (B.OaplTensor * len(kw))(*[_set(B.OaplTensor(at(1 + i), at(100 + i), 1000, 0, 0), k) for i, k in enumerate(kw)])


@pytest.mark.parametrize("kw, want", [
    (dict(n=-1), INVALID), (dict(data=0), INVALID), (dict(type=3), INVALID), (dict(data=at(1, 1)), MISALIGNED),
    (dict(n=1 << 62), UNSUPPORTED)])
def test_tensor_list(L, kw, want):
    t = _tensors({}, kw)
    assert L.oapl_grad_norm(t, 2, 1.0, at(90), at(91), None, at(92), 1 << 40, ST) == want
    assert L.oapl_grad_clip(t, 2, 1.0, at(90), 1.0, ST) == want


def test_gradient_norm_and_clip_arguments(L):
    t = _tensors({}, {})
    f = lambda t=t, c=2, s=1.0, sq=at(90), n=at(91), ws=at(92), size=1 << 40: L.oapl_grad_norm(t, c, s, sq, n, None, ws, size, ST)  # noqa: E731
    assert f(t=None) == f(c=0) == f(c=-1) == f(s=NAN) == f(sq=None, n=None) == f(ws=None) == INVALID
    assert f(ws=at(92, 8)) == f(sq=at(90, 2)) == MISALIGNED
    need = L.oapl_grad_norm_workspace_bytes(2)
    assert need > 0 and f(size=need - 1) == SMALL
    assert L.oapl_grad_norm_workspace_bytes(0) == 0 and L.oapl_grad_norm_workspace_bytes(1000) > need
    g = lambda t=t, c=2, s=1.0, sq=at(90), clip=1.0: L.oapl_grad_clip(t, c, s, sq, clip, ST)  # noqa: E731
    assert g(t=None) == g(c=0) == g(s=INF) == g(sq=None) == g(clip=0.0) == g(clip=-1.0) == g(clip=NAN) == g(clip=INF) == INVALID
    assert g(sq=at(90, 1)) == MISALIGNED
    assert g(t=_tensors({}, dict(out=0))) == g(t=_tensors({}, dict(out_type=7))) == INVALID
    assert g(t=_tensors(dict(out=at(1), out_type=2))) == INVALID           # in place in another type
    assert g(t=_tensors(dict(out=at(1, 4)))) == INVALID                    # partly over itself
    assert g(t=_tensors(dict(out=at(100, 2), out_type=2)), c=1) == MISALIGNED


def _logits(**kw):
    return _set(B.OaplLogits(at(1), 64, 1000, 1000, 0, None, None, 1.0), kw)


def _adjust(**kw):
    return _set(B.OaplAdjust(at(2), 5000, at(3), at(4), at(5), at(6), at(7), at(8), at(9), 10, at(10), 32, 64, None), kw)


@pytest.mark.parametrize("kw, want", [
    (dict(T=-1), INVALID), (dict(biases=-1), INVALID), (dict(spans=0), INVALID), (dict(tokens=0), INVALID),
    (dict(tokens=0, spans=0, T=0), INVALID), (dict(bias_id=0), INVALID), (dict(bias=0), INVALID), (dict(ld_allowed=31), INVALID),
    (dict(allowed_rows=0), INVALID), (dict(allowed_rows=63), INVALID), (dict(allowed=0, allowed_row=at(11)), INVALID),
    (dict(tokens=at(2, 2)), MISALIGNED), (dict(spans=at(3, 4)), MISALIGNED), (dict(repetition=at(4, 1)), MISALIGNED),
    (dict(bias_start=at(7, 4)), MISALIGNED), (dict(allowed=at(10, 2)), MISALIGNED)])
def test_adjust_struct(L, kw, want):
    assert L.oapl_logits_adjust(_logits(), _adjust(**kw), at(20), 1000, None, ST) == want
    assert L.oapl_logits_adjust_bwd(_logits(), _adjust(**kw), at(20), 1000, at(21), 1000, None, ST) == want


def test_adjust_arguments(L):
    f = lambda l=_logits(), a=_adjust(), out=at(20), ld=1000: L.oapl_logits_adjust(l, a, out, ld, None, ST)  # noqa: E731
    assert f(l=None) == f(a=None) == f(out=None) == f(ld=999) == f(l=_logits(V=0)) == f(l=_logits(type=4)) == INVALID
    assert f(out=at(20, 1)) == MISALIGNED
    assert f(out=at(1), ld=1001) == f(out=at(1, 2)) == INVALID             # over the logits only row by row
    big = _logits(N=2 * 10 ** 9, V=152064, ld=152064)
    assert f(l=big, a=_adjust(allowed=0), ld=152064) in (INVALID, UNSUPPORTED)
    g = lambda l=_logits(), a=_adjust(), d=at(20), ld=1000, o=at(21), lo=1000: L.oapl_logits_adjust_bwd(l, a, d, ld, o, lo, None, ST)  # noqa: E731
    assert g(l=None) == g(a=None) == g(d=None) == g(o=None) == g(ld=999) == g(lo=999) == INVALID
    assert g(d=at(20, 1)) == g(o=at(21, 1)) == MISALIGNED
    assert g(o=at(20, 2)) == g(o=at(1, 2)) == INVALID


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        B.make_lookup(torch.zeros(4, dtype=torch.int32), 8)
    with pytest.raises(TypeError):
        B.make_residual(x)
    with pytest.raises(TypeError):
        B.make_tensor_list([x])
    with pytest.raises(ValueError):
        B.make_tensor_list([])
