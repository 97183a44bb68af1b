"""Operators around the attention, what needs no GPU: refusals of the C-ABI before anything is launched, frequencies,
what the native argument path leaves to the binding."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2502_07864_amd import layer, mla

OK, E_NULL, E_SHAPE, E_UNSUP, E_WS = 0, -1, -2, -3, -4
F32, BF16, FP8 = 0, 1, 2
P = 0x10000   # a non-NULL pointer value, never used: every call below is refused


@pytest.fixture(scope="module")
def L():
    return mla.lib()


def norm(L, x=P, residual=None, weight=P, residual_out=None, y=P, codes=None, scales=None, T=4, D=256, pitch=256, eps=1e-6, io=BF16):
    return L.mla_rms_norm(x, residual, weight, residual_out, y, codes, scales, T, D, pitch, eps, io, None)


@pytest.mark.parametrize("kw, want", [
    (dict(x=None), E_NULL), (dict(y=None), E_NULL), (dict(y=None, codes=P), E_NULL), (dict(scales=P), E_NULL),
    (dict(residual=P), E_NULL), (dict(residual_out=P), E_NULL),
    (dict(T=0), E_SHAPE), (dict(D=0, pitch=0), E_SHAPE), (dict(pitch=255), E_SHAPE), (dict(eps=-1.0), E_SHAPE), (dict(eps=math.nan), E_SHAPE),
    (dict(io=FP8), E_UNSUP), (dict(io=7), E_UNSUP), (dict(D=32769, pitch=32769), E_UNSUP), (dict(T=1 << 24), E_UNSUP)])
def test_norm_refusals(L, kw, want):
    assert norm(L, **kw) == want


def test_quantize_refusals(L):
    assert L.mla_quantize_rows(None, P, P, 4, 256, 256, BF16, None) == E_NULL
    assert L.mla_quantize_rows(P, P, None, 4, 256, 256, BF16, None) == E_NULL
    assert L.mla_quantize_rows(P, P, P, 4, 256, 255, BF16, None) == E_SHAPE
    assert L.mla_quantize_rows(P, P, P, 4, 256, 256, FP8, None) == E_UNSUP
    assert L.mla_quantize_weights(P, None, P, 4, 256, BF16, None) == E_NULL
    assert L.mla_quantize_weights(P, P, P, 0, 256, BF16, None) == E_SHAPE
    assert L.mla_quantize_weights(P, P, P, 4, 256, FP8, None) == E_UNSUP


def gemm(L, a=P, sa=P, w=P, sw=P, out=P, ws=P, ws_bytes=1 << 40, M=4, N=64, K=256, dt=BF16, flags=0):
    return L.mla_gemm_fp8(a, sa, w, sw, out, ws, ws_bytes, M, N, K, dt, flags, None)


@pytest.mark.parametrize("kw, want", [
    (dict(a=None), E_NULL), (dict(sa=None), E_NULL), (dict(w=None), E_NULL), (dict(sw=None), E_NULL), (dict(out=None), E_NULL),
    (dict(M=0), E_SHAPE), (dict(N=-1), E_SHAPE), (dict(K=0), E_SHAPE),
    (dict(K=24), E_UNSUP), (dict(dt=FP8), E_UNSUP), (dict(a=P + 8), E_UNSUP), (dict(w=P + 1), E_UNSUP), (dict(flags=2), E_UNSUP), (dict(K=(1 << 23) + 16), E_UNSUP),
    (dict(M=(1 << 30) + 1), E_UNSUP), (dict(N=0x7FFFFFFF), E_UNSUP), (dict(M=1 << 30, N=1 << 30, K=16), E_UNSUP)])
def test_gemm_refusals(L, kw, want):
    assert gemm(L, **kw) == want


def test_gemm_workspace(L):
    assert L.mla_gemm_fp8_workspace_bytes(0x7FFFFFFF, 64, 64) == 0 and L.mla_gemm_fp8_workspace_bytes(0, 64, 64) == 0 and L.mla_gemm_fp8_workspace_bytes(4, 64, -1) == 0
    for M in (1, 16, 61, 500, 4000):
        for N in (320, 576, 3584):
            for K in (256, 4096):
                need = L.mla_gemm_fp8_workspace_bytes(M, N, K)
                if need:      # sizes that want scratch say so when it is missing, short or off 16 bytes
                    assert gemm(L, ws=None, ws_bytes=0, M=M, N=N, K=K) == E_WS
                    assert gemm(L, ws_bytes=need - 1, M=M, N=N, K=K) == E_WS
                    assert gemm(L, ws=P + 4, M=M, N=N, K=K) == E_WS


def rope(L, q=P, pos=P, freq=P, qn=P, qr=P, T=4, H=2, dn=128, dr=64, pitch=384, gain=1.0, layout=0, io=BF16):
    return L.mla_rope_queries(q, pos, freq, qn, qr, T, H, dn, dr, pitch, gain, layout, io, None)


@pytest.mark.parametrize("kw, want", [
    (dict(q=None), E_NULL), (dict(pos=None), E_NULL), (dict(freq=None), E_NULL), (dict(qn=None), E_NULL), (dict(qr=None), E_NULL),
    (dict(T=0), E_SHAPE), (dict(H=0), E_SHAPE), (dict(dn=-1), E_SHAPE), (dict(dr=0), E_SHAPE), (dict(dr=63), E_SHAPE),
    (dict(pitch=383), E_SHAPE), (dict(gain=math.nan), E_SHAPE),
    (dict(layout=2), E_UNSUP), (dict(io=FP8), E_UNSUP), (dict(dr=258, pitch=4096), E_UNSUP), (dict(T=1 << 24), E_UNSUP),
    (dict(H=1 << 23, pitch=1 << 40), E_UNSUP)])
def test_rope_refusals(L, kw, want):
    assert rope(L, **kw) == want


def store(L, rows=P, pos=P, freq=P, w=None, kv=P, scale=None, table=P, B=2, new=3, d_c=512, d_rope=64, pitch=576, page=64, pages=8,
          width=4, gain=1.0, layout=0, eps=1e-6, io=BF16, cache=BF16):
    return L.mla_cache_store(rows, pos, freq, w, kv, scale, table, B, new, d_c, d_rope, pitch, page, pages, width, gain, layout, eps, io, cache, None)


@pytest.mark.parametrize("kw, want", [
    (dict(rows=None), E_NULL), (dict(pos=None), E_NULL), (dict(freq=None), E_NULL), (dict(kv=None), E_NULL), (dict(table=None), E_NULL),
    (dict(cache=FP8), E_NULL), (dict(scale=P), E_SHAPE), (dict(B=0), E_SHAPE), (dict(new=0), E_SHAPE), (dict(d_c=0), E_SHAPE),
    (dict(d_rope=63), E_SHAPE), (dict(d_rope=-2), E_SHAPE), (dict(pitch=575), E_SHAPE), (dict(page=0), E_SHAPE), (dict(pages=0), E_SHAPE),
    (dict(width=0), E_SHAPE), (dict(width=1 << 26, page=64), E_SHAPE), (dict(gain=math.nan), E_SHAPE), (dict(eps=-1.0), E_SHAPE),
    (dict(layout=-1), E_UNSUP), (dict(io=FP8), E_UNSUP), (dict(cache=5), E_UNSUP), (dict(d_c=1000, pitch=2000), E_UNSUP),
    (dict(d_rope=258, d_c=512, pitch=2000), E_UNSUP), (dict(d_c=0x7FFFFFFF, pitch=1 << 40), E_UNSUP), (dict(B=1 << 20, new=1 << 10), E_UNSUP)])
def test_store_refusals(L, kw, want):
    assert store(L, **kw) == want


# ------------------------------------------------------------------ frequencies

def test_plain_and_linear_frequencies():
    f, g = layer.rope_frequencies(64, device="cpu")
    want = np.array([10000.0 ** (-2 * i / 64) for i in range(32)])
    np.testing.assert_allclose(f.numpy(), want, rtol=1e-14)
    assert g == 1.0 and f.dtype == torch.float64
    f2, g2 = layer.rope_frequencies(64, scaling="linear", factor=4.0, device="cpu")
    np.testing.assert_allclose(f2.numpy(), want / 4, rtol=1e-14)
    assert g2 == 1.0


@pytest.mark.parametrize("d, base, factor, original", [(64, 10000.0, 40.0, 4096), (128, 500000.0, 8.0, 8192), (32, 10000.0, 1.0, 2048)])
def test_yarn_frequencies(d, base, factor, original):
    """Against the definition pair by pair: turns within the original length decide."""
    f, g = layer.rope_frequencies(d, base, "yarn", factor, original, 32.0, 1.0, device="cpu")
    theta = np.array([base ** (-2 * i / d) for i in range(d // 2)])
    turns = original * theta / (2 * np.pi)
    f = f.numpy()
    fast, slow = turns >= 32.0, turns < 1.0
    # the ends of the ramp are rounded outwards to whole pairs: pairs beyond them are exactly one or the other
    np.testing.assert_allclose(f[fast][:-1], theta[fast][:-1], rtol=1e-13)
    np.testing.assert_allclose(f[slow][1:], theta[slow][1:] / factor, rtol=1e-13)
    assert (f <= theta * (1 + 1e-13)).all() and (f >= theta / factor * (1 - 1e-13)).all()
    w = (f / theta - 1 / factor) / (1 - 1 / factor) if factor > 1 else None
    if w is not None:       # share of the unscaled frequency: falls linearly with the pair's index
        inside = w[(w > 1e-9) & (w < 1 - 1e-9)]
        assert len(inside) >= 3 and np.abs(np.diff(inside, 2)).max() < 1e-9 and (np.diff(inside) < 0).all()
    assert abs(g - (0.1 * math.log(factor) + 1.0)) < 1e-6


@pytest.mark.parametrize("kw", [dict(d_rope=63), dict(d_rope=0), dict(base=1.0), dict(base=math.inf), dict(scaling="linear", factor=0.5),
                                dict(scaling="yarn", factor=math.nan), dict(scaling="yarn", factor=2.0, original=0),
                                dict(scaling="yarn", factor=2.0, beta_fast=0.5), dict(scaling="yarn", factor=2.0, beta_slow=0.0)])
def test_frequency_refusals(kw):
    with pytest.raises(mla.MlaError):
        layer.rope_frequencies(**{"d_rope": 64, "device": "cpu", **kw})


def test_unknown_scaling():
    with pytest.raises(ValueError, match="scaling"):
        layer.rope_frequencies(64, scaling="ntk", device="cpu")


# ------------------------------------------------------------------ the binding

@pytest.mark.parametrize("bad", [torch.zeros(2, 128), torch.zeros(2, 128, dtype=torch.float64), None, 3, "x", torch.zeros(128, 2).t()])
def test_arguments_it_does_not_take_are_left_to_the_binding(bad):
    mla.lib()
    x = torch.zeros(2, 128)
    f = mla._fast
    assert f.rms_norm(bad, None, 1e-6, None, None, x, None, None) is None and f.rms_norm(x) is None
    assert f.quantize_rows(bad, x, x) is None
    assert f.gemm_fp8(bad, x, x, x, x, None, 0) is None
    assert f.rope_queries(bad, x, x, 1.0, 0, x, x) is None
    assert f.cache_store(bad, x, x, x, x, 64, 1.0, 0, None, 1e-6, None) is None


def test_the_checks_of_the_binding():
    x = torch.zeros(2, 128)
    with pytest.raises(ValueError, match="GPU tensor"):
        layer.rms_norm(x)
    with pytest.raises(ValueError, match=r"\[T, D\]"):
        layer.rms_norm(torch.zeros(128))
    with pytest.raises(ValueError, match="GPU tensor"):
        layer.quantize_rows(x)
    with pytest.raises(ValueError, match=r"\[M, K\]"):
        layer.gemm_fp8(x, x, torch.zeros(4, 64), x)
    with pytest.raises(TypeError, match="float8"):
        layer.gemm_fp8(x, x, x, x)
    with pytest.raises(TypeError, match="float64"):
        layer.rope_queries(torch.zeros(2, 1, 64), torch.zeros(2, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(ValueError, match="rows must be"):
        layer.cache_store(x, x, x, x, x, 64)
