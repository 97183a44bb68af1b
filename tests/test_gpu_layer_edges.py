"""Operators around the attention at the edges of their definitions."""
import math

import pytest
import torch

from paper_2502_07864_amd import layer, mla
from test_gpu_layer import BF, DEV, F32, FAST_DROP, FAST_NORM, FP8, ROUND, blocks, dequantised, near, operands, ref_norm, rnd, the_calls

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ codes

def middles():
    """The numbers half way between two neighbouring normal codes, of both signs."""
    m = torch.arange(8, 16, dtype=torch.float64)
    t = torch.stack([(2 * m + 1) / 16 * 2.0 ** e for e in range(-6, 9)]).flatten()
    t = t[t < 448]
    return torch.cat((t, -t))


def rows_of_middles(n, seed):
    """[n, 256] in fp32: in every block of 128 columns 448 s and products t s with the middles t, all exact, s of 16 bits."""
    g = torch.Generator().manual_seed(seed)
    t = middles()
    at = torch.randint(0, t.numel(), (n, 2, 128), generator=g)
    t = t[at]
    t[..., 0] = 448.0
    s = torch.randint(1 << 15, 1 << 16, (n, 2, 1), generator=g).double() * 2.0 ** torch.randint(-40, 20, (n, 2, 1), generator=g).double()
    x = t * s
    assert torch.equal(x.float().double(), x)
    return x.float().view(n, 256), t.view(n, 256), s.view(n, 2)


def test_a_quotient_in_the_middle_goes_to_the_even_code():
    x, t, s = rows_of_middles(2000, 1)
    want = t.float().to(FP8).view(torch.uint8)
    for width in (256, 255):                                    # in whole vectors and in pieces
        codes, scales = layer.quantize_rows(x[:, :width].contiguous().to(DEV))
        assert torch.equal(scales.t().cpu().double(), s)
        assert torch.equal(codes.view(torch.uint8).cpu(), want[:, :width])


def test_a_weights_quotient_in_the_middle_goes_to_the_even_code():
    g = torch.Generator().manual_seed(3)
    x, t, _ = rows_of_middles(128 * 9, 2)
    s = torch.randint(1 << 15, 1 << 16, (9, 2), generator=g).double() * 2.0 ** -20
    w = (t.view(9, 128, 2, 128) * s[:, None, :, None]).view(128 * 9, 256)
    codes, scales = layer.quantize_weights(w.float().to(DEV))
    assert torch.equal(scales.cpu().double(), s)
    assert torch.equal(codes.view(torch.uint8).cpu(), t.float().to(FP8).view(torch.uint8))


@pytest.mark.parametrize("io", [BF, F32])
@pytest.mark.parametrize("D", [1024, 1001])
def test_codes_are_those_of_the_quotient(io, D):
    """Every code of many rows is the fp32 quotient's, rounded to nearest even; zeros keep their signs."""
    x = rnd(3000, D, dtype=io, loud=True)
    x[:, 7] = -0.0
    codes, scales = layer.quantize_rows(x)
    unit = scales.cpu().repeat_interleave(128, 0)[:D].t()
    assert torch.equal(codes.view(torch.uint8).cpu(), (x.cpu().float() / unit).to(FP8).view(torch.uint8))


def test_codes_of_a_block_with_an_infinity():
    """Its scale is infinite, its finite values' codes are zeros, the infinity's is not a number; other blocks are as they were."""
    x = rnd(4, 512, dtype=F32)
    want, want_s = layer.quantize_rows(x)
    x[1, 200] = math.inf
    x[2, 300] = -math.inf
    codes, scales = layer.quantize_rows(x)
    nan = torch.isnan(codes.float())
    assert nan.sum() == 2 and nan[1, 200] and nan[2, 300]
    assert torch.isinf(scales[1, 1]) and torch.isinf(scales[2, 2]) and torch.isinf(scales).sum() == 2
    assert not codes.float()[1, 128:256][~nan[1, 128:256]].any() and not codes.float()[2, 256:384][~nan[2, 256:384]].any()
    same = torch.ones(4, 512, dtype=torch.bool, device=DEV)
    same[1, 128:256], same[2, 256:384] = False, False
    assert torch.equal(codes.view(torch.uint8)[same], want.view(torch.uint8)[same])


@pytest.mark.parametrize("io", [BF, F32])
@pytest.mark.parametrize("layout", [0, 1])
def test_cache_rows_have_the_same_bits_at_any_address(io, layout):
    """Rows that lie on 16 bytes and rows that do not take different kernels; infinities, NaN and negative zeros among them."""
    n, d_c, row = 60, 512, 576
    rows = rnd(1, n, row, dtype=io, loud=True)
    rows[0, 3, 17], rows[0, 9, 100], rows[0, 20, 511] = math.inf, -math.inf, math.nan
    rows[0, 5, 40:90] = -0.0
    rows[0, 6] = -0.0
    rows[0, 9, 200:300] = -0.0
    wide = torch.zeros((1, n, row + 3), dtype=io, device=DEV)
    wide[..., 1:1 + row] = rows
    freq, gain = layer.rope_frequencies(64)
    pos, table = torch.arange(n, dtype=torch.int32, device=DEV).view(1, n), torch.tensor([[1]], dtype=torch.int32, device=DEV)
    got = []
    for x in (rows, wide[..., 1:1 + row]):
        kv, scale = torch.zeros((2, 64, row), dtype=torch.uint8, device=DEV), torch.zeros((2, 64), device=DEV)
        layer.cache_store(x, pos, freq, kv, table, d_c, gain, layout, kv_scale=scale)
        kv = torch.where((kv & 0x7F) == 0x7F, torch.full_like(kv, 0x7F), kv)           # (a NaN's sign says nothing)
        got.append((kv, scale))
    assert torch.equal(got[0][0], got[1][0])
    assert torch.equal(got[0][1].view(torch.int32), got[1][1].view(torch.int32))
    kv, scale = got[0][0][1].view(FP8).float(), got[0][1][1]
    for r, c in ((3, 17), (9, 100)):
        assert torch.isinf(scale[r]) and torch.isnan(kv[r, c]) and not kv[r, :c].any() and not kv[r, c + 1:].any()
    assert torch.isnan(scale[20]) and torch.isnan(kv[20]).all()


# ------------------------------------------------------------------ norm

def test_the_sum_may_take_the_place_of_x():
    """residual_out is x itself, with the codes and without, in whole vectors and in pieces."""
    for D in (4096, 1001):
        x, r, w = rnd(70, D, dtype=BF), rnd(70, D, dtype=BF, seed=3), rnd(D, dtype=BF, seed=4)
        want, want_s = layer.rms_norm(x, w, residual=r)
        codes, scales, _, _ = layer.rms_norm_fp8(x, w, residual=r)
        a, b = x.clone(), x.clone()
        y, s = layer.rms_norm(a, w, residual=r, residual_out=a)
        assert s is a and torch.equal(a, want_s) and torch.equal(y, want)
        near(a, ref_norm(x, w, 1e-6, r)[0], ROUND[BF], 2.0 ** -24 * (x.double().abs() + r.double().abs()))
        codes2, scales2, s2, _ = layer.rms_norm_fp8(b, w, residual=r, residual_out=b)
        assert torch.equal(s2, want_s) and torch.equal(codes2.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(scales2, scales)


# ------------------------------------------------------------------ products whose depth is shared out

# sizes at which the product of either kind of sums (fast or not) writes partial sums to the workspace
SHARED = [(136, 6088, 7184, False), (146, 6006, 8448, False), (1032, 1208, 9808, True), (2877, 171, 14352, True)]


@pytest.mark.parametrize("M, N, K, fast", SHARED)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_shares_of_the_depth(M, N, K, fast, dtype):
    """Against 64 bits; the partial sums go through the workspace, and around it and the outputs nothing changes; five times
    the same bits, whatever the workspace held."""
    a, sa, w, sw = operands(M, N, K)
    need = layer.gemm_fp8_workspace_bytes(M, N, K)
    assert need >= 2 * 4 * M * N
    room = torch.full((M * N + 512,), 7.0, dtype=dtype, device=DEV)
    out = room[256:256 + M * N].view(M, N)
    scratch = torch.full((need + 512,), 0xAB, dtype=torch.uint8, device=DEV)
    flags = layer.GEMM_FAST_SUMS if fast else 0
    layer.gemm_fp8(a, sa, w, sw, out=out, workspace=scratch[256:256 + need], flags=flags)
    A, W = dequantised(a, sa, w, sw)
    want, size = torch.mm(A, W.t().contiguous()), torch.mm(A.abs(), W.abs().t().contiguous())
    near(out, want, ROUND[dtype], ((FAST_DROP if fast else 0.0) + (140 + blocks(K)) * 2.0 ** -24) * size)
    if fast:
        assert (out.double() - want).norm() <= (FAST_NORM + (2.0 ** -9 if dtype == BF else 0.0)) * want.norm()
    assert (scratch[256:256 + 4 * M * N] != 0xAB).any()
    assert (scratch[:256] == 0xAB).all() and (scratch[256 + need:] == 0xAB).all()
    assert (room[:256] == 7).all() and (room[256 + M * N:] == 7).all()
    first = out.clone()
    for fill in (0, 0x7F, 0xFF, 0x55):
        scratch.fill_(fill)
        layer.gemm_fp8(a, sa, w, sw, out=out, workspace=scratch[256:256 + need], flags=flags)
        assert torch.equal(out, first)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("M, N, K, fast", SHARED[1:3])
def test_a_workspace_is_checked_or_made(M, N, K, fast, native, monkeypatch):
    """One that is short or off 16 bytes is refused and nothing is written; without one the binding brings its own."""
    mla.lib()
    if not native:
        monkeypatch.setattr(mla, "_fast", None)
    a, sa, w, sw = operands(M, N, K)
    need = layer.gemm_fp8_workspace_bytes(M, N, K)
    assert need > 0
    flags = layer.GEMM_FAST_SUMS if fast else 0
    out = torch.zeros((M, N), dtype=BF, device=DEV)
    room = torch.empty(need + 16, dtype=torch.uint8, device=DEV)
    for ws in (room[:need - 1], room[8:8 + need], room[:0]):
        with pytest.raises(mla.MlaError) as e:
            layer.gemm_fp8(a, sa, w, sw, out=out, workspace=ws, flags=flags)
        assert e.value.status == -4
    torch.cuda.synchronize()
    assert not out.any()
    want = layer.gemm_fp8(a, sa, w, sw, workspace=room[:need], flags=flags)
    assert layer.gemm_fp8(a, sa, w, sw, out=out, flags=flags) is out and torch.equal(out, want)


# ------------------------------------------------------------------ outputs of another type

OTHER = {
    "norm": [dict(out=torch.float16), dict(out=torch.int16), dict(residual_out=torch.float16), dict(codes=torch.int8), dict(codes=torch.bool),
             dict(codes=torch.float8_e5m2), dict(scales=torch.int32)],
    "quantize": [dict(codes=torch.int8), dict(codes=torch.float8_e5m2), dict(scales=torch.int32)],
    "rope": [dict(q_nope=torch.float16), dict(q_rope=torch.float16), dict(q_rope=torch.int16)],
}


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", list(OTHER))
def test_outputs_of_another_type_are_refused(name, native, monkeypatch):
    """Their size would do; their type is not what is written there.  Nothing is written."""
    mla.lib()
    f, args, outputs = the_calls()[name]
    if not native:
        monkeypatch.setattr(mla, "_fast", None)
    for case in OTHER[name]:
        a = {**args, **{k: args[k].view(torch.uint8).clone().view(t) for k, t in case.items()}}
        with pytest.raises((ValueError, TypeError)):
            f(**a)
        torch.cuda.synchronize()
        for k in outputs:
            assert not a[k].view(torch.uint8).any(), (case, k)
