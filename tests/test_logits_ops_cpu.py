"""Refusals of the calls on logits in memory and on 8-bit matrices: all are made on the host, before any
CUDA call, so they are tested without a GPU (the addresses are never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2602_19362_b200 import binding as B, build

OUT, ST = ctypes.c_void_p(0x2000), ctypes.c_void_p(0)
INVALID, MISALIGNED, UNSUPPORTED = -1, -2, -4


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def _logits(**kw):
    p = B.OaplLogits(0x1000, 64, 1000, 1000, 0, 0x3000, 0x4000, 1.0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _scaled(**kw):
    m = B.OaplScaled(0x1000, 0x2000, 256, 512, 512, 1, 256, 3, 1)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


@pytest.mark.parametrize("kw, want", [
    (dict(logits=0), INVALID), (dict(N=0), INVALID), (dict(N=-3), INVALID), (dict(V=0), INVALID), (dict(ld=999), INVALID),
    (dict(type=3), INVALID), (dict(type=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(targets=0), INVALID),
    (dict(logits=0x1001), MISALIGNED), (dict(type=2, logits=0x1002), MISALIGNED), (dict(N=3 * 10 ** 9), UNSUPPORTED),
    (dict(V=2 * 10 ** 9 + 1, ld=3 * 10 ** 9), UNSUPPORTED)])
def test_logits_struct(L, kw, want):
    p = _logits(**kw)
    assert L.oapl_logits_logprobs(p, OUT, OUT, OUT, 4, OUT, OUT, None, ST) == want
    assert L.oapl_logits_logprobs_bwd(p, OUT, OUT, OUT, OUT, 0, None, None, OUT, 1 << 40, ST) == want


def test_logprobs_outputs(L):
    f = L.oapl_logits_logprobs
    p = _logits()
    assert f(None, OUT, OUT, OUT, 0, None, None, None, ST) == INVALID
    assert f(p, None, None, None, 0, None, None, None, ST) == INVALID     # nothing asked for
    assert f(p, OUT, OUT, OUT, -1, OUT, OUT, None, ST) == INVALID
    assert f(p, OUT, OUT, OUT, 33, OUT, OUT, None, ST) == INVALID
    assert f(p, OUT, OUT, OUT, 5, None, None, None, ST) == INVALID        # alternatives without a place
    assert f(p, OUT, OUT, OUT, 0, OUT, None, None, ST) == INVALID


def test_logprobs_gradient_arguments(L):
    f = L.oapl_logits_logprobs_bwd
    p = _logits()
    assert f(None, OUT, OUT, OUT, OUT, 0, None, None, OUT, 1000, ST) == INVALID
    assert f(p, None, OUT, OUT, OUT, 0, None, None, OUT, 1000, ST) == INVALID    # no log-sum-exp
    assert f(p, OUT, OUT, OUT, OUT, 0, None, None, None, 1000, ST) == INVALID
    assert f(p, OUT, OUT, OUT, OUT, 0, None, None, OUT, 999, ST) == INVALID
    assert f(p, OUT, OUT, None, None, 0, None, None, OUT, 1000, ST) == INVALID   # no gradient given
    assert f(p, OUT, None, OUT, OUT, 0, None, None, OUT, 1000, ST) == INVALID    # entropy's gradient without the entropy
    assert f(p, OUT, OUT, OUT, OUT, 4, None, None, OUT, 1000, ST) == INVALID
    assert f(p, OUT, OUT, OUT, OUT, 4, OUT, None, OUT, 1000, ST) == INVALID
    assert f(p, OUT, OUT, OUT, OUT, 0, OUT, OUT, OUT, 1000, ST) == INVALID
    assert f(p, OUT, OUT, OUT, OUT, 33, OUT, OUT, OUT, 1000, ST) == INVALID
    assert f(p, OUT, OUT, OUT, OUT, 0, None, None, ctypes.c_void_p(0x2001), 1000, ST) == MISALIGNED
    # in place with another stride would overwrite logits that are still to be read
    assert f(p, OUT, OUT, OUT, OUT, 0, None, None, ctypes.c_void_p(p.logits), 1001, ST) == INVALID
    # more rows x spans than a grid holds
    big = _logits(N=2 * 10 ** 9, V=152064, ld=152064)
    assert f(big, OUT, OUT, OUT, OUT, 0, None, None, OUT, 152064, ST) == UNSUPPORTED


@pytest.mark.parametrize("kw, want", [
    (dict(data=0), INVALID), (dict(scale=0), INVALID), (dict(rows=0), INVALID), (dict(cols=0), INVALID),
    (dict(ld=500), INVALID), (dict(type=0), INVALID), (dict(type=5), INVALID), (dict(block_rows=64), INVALID),
    (dict(block_rows=0), INVALID), (dict(scale_row_stride=-1), INVALID), (dict(scale_col_stride=-1), INVALID),
    (dict(data=0x1008), MISALIGNED), (dict(ld=520), MISALIGNED), (dict(scale=0x2002), MISALIGNED),
    (dict(rows=3 * 10 ** 9), UNSUPPORTED)])
def test_scaled_struct(L, kw, want):
    m = _scaled(**kw)
    assert L.oapl_quantize(OUT, 0, 256, 512, 512, m, 0, ST) == want
    assert L.oapl_scaled_matmul(m, _scaled(), OUT, 0, 256, 0, None, ST) == want
    assert L.oapl_scaled_matmul(_scaled(), m, OUT, 0, 1 << 40, 0, None, ST) == want


def test_quantize_arguments(L):
    f = L.oapl_quantize
    m = _scaled()
    assert f(None, 0, 256, 512, 512, m, 0, ST) == INVALID
    assert f(OUT, 3, 256, 512, 512, m, 0, ST) == INVALID
    assert f(OUT, 0, 256, 512, 511, m, 0, ST) == INVALID
    assert f(OUT, 0, 255, 512, 512, m, 0, ST) == INVALID
    assert f(OUT, 0, 256, 512, 512, m, 1, ST) == INVALID          # turned: out would have to be 512 x 256
    assert f(OUT, 0, 256, 512, 512, m, 4, ST) == INVALID
    assert f(OUT, 0, 256, 512, 512, None, 0, ST) == INVALID
    assert f(ctypes.c_void_p(0x2001), 0, 256, 512, 512, m, 0, ST) == MISALIGNED
    assert f(ctypes.c_void_p(0x2002), 2, 256, 512, 512, m, 0, ST) == MISALIGNED


def test_scaled_matmul_arguments(L):
    f = L.oapl_scaled_matmul
    m = _scaled()
    assert f(None, m, OUT, 0, 256, 0, None, ST) == INVALID
    assert f(m, None, OUT, 0, 256, 0, None, ST) == INVALID
    assert f(m, m, None, 0, 256, 0, None, ST) == INVALID
    assert f(m, m, OUT, 3, 256, 0, None, ST) == INVALID
    assert f(m, m, OUT, 0, 255, 0, None, ST) == INVALID
    assert f(m, _scaled(cols=500), OUT, 0, 256, 0, None, ST) == INVALID
    assert f(m, m, ctypes.c_void_p(0x2001), 0, 256, 0, None, ST) == MISALIGNED
    assert f(m, m, ctypes.c_void_p(0x2002), 2, 256, 0, None, ST) == MISALIGNED


def test_binding_refuses_host_tensors_and_wrong_types():
    z = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        B.make_logits(z)
    with pytest.raises(TypeError):
        B.make_logits(z.to(torch.float64))
    with pytest.raises(TypeError):
        B.make_scaled(torch.zeros(4, 16).to(torch.float8_e4m3fn), torch.ones(4, 1), 1)
    with pytest.raises(TypeError):
        B.oapl_quantize(z, None)
