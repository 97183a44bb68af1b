"""Masked attention and moved rows, what needs no GPU: refusals of the C-ABI before anything is launched, workspace sizes, what the
binding refuses."""
import math

import pytest
import torch

from paper_2502_07864_amd import layer, mla

OK, E_NULL, E_SHAPE, E_UNSUP, E_WS = 0, -1, -2, -3, -4
F32, BF16, FP8 = 0, 1, 2
P = 0x10000   # a non-NULL pointer value, never used: every call below is refused
BIG = 1 << 50


@pytest.fixture(scope="module")
def L():
    return mla.lib()


COMMON = [
    (dict(q=None), E_NULL), (dict(qr=None), E_NULL), (dict(kv=None), E_NULL), (dict(table=None), E_NULL), (dict(lens=None), E_NULL),
    (dict(out=None), E_NULL), (dict(cache=FP8), E_NULL), (dict(kv_scale=P), E_SHAPE),
    (dict(B=0), E_SHAPE), (dict(T=0), E_SHAPE), (dict(H=-1), E_SHAPE), (dict(d_c=0), E_SHAPE), (dict(d_rope=-8), E_SHAPE), (dict(page=0), E_SHAPE),
    (dict(pages=0), E_SHAPE), (dict(width=0), E_SHAPE), (dict(width=1 << 30), E_SHAPE), (dict(scale=math.nan), E_SHAPE),
    (dict(io=FP8), E_UNSUP), (dict(io=9), E_UNSUP), (dict(cache=7), E_UNSUP), (dict(cache=F32), E_UNSUP), (dict(d_c=520), E_UNSUP),
    (dict(d_c=12), E_UNSUP), (dict(d_rope=72), E_UNSUP), (dict(d_rope=4), E_UNSUP), (dict(B=65536), E_UNSUP), (dict(T=32, H=257), E_UNSUP),
    (dict(flags=2), E_UNSUP), (dict(flags=4), E_UNSUP), (dict(flags=9), E_UNSUP),
    (dict(ws=None), E_WS), (dict(ws_bytes=64), E_WS), (dict(ws=P + 128), E_WS)]


def tree(L, q=P, qr=P, kv=P, kv_scale=None, table=P, lens=P, mask=P, pitch=None, out=P, lse=None, ws=P, ws_bytes=BIG, B=1, T=4, H=32, d_c=512,
         d_rope=64, page=64, pages=200, width=100, scale=0.1, io=BF16, cache=BF16, flags=0):
    return L.mla_decode_paged_tree(q, qr, kv, kv_scale, table, lens, mask, T if pitch is None else pitch, out, lse, ws, ws_bytes, B, T, H, d_c,
                                   d_rope, page, pages, width, scale, io, cache, flags, None)


@pytest.mark.parametrize("kw, want", COMMON + [(dict(mask=None), E_NULL), (dict(T=65), E_UNSUP), (dict(pitch=3), E_SHAPE), (dict(pitch=-1), E_SHAPE)])
def test_tree_refusals(L, kw, want):
    assert tree(L, **kw) == want


def window(L, q=P, qr=P, kv=P, kv_scale=None, table=P, lens=P, out=P, lse=None, ws=P, ws_bytes=BIG, B=1, T=4, H=32, d_c=512, d_rope=64, page=64,
           pages=200, width=100, window=2000, sinks=4, scale=0.1, io=BF16, cache=BF16, flags=0):
    return L.mla_decode_paged_window(q, qr, kv, kv_scale, table, lens, out, lse, ws, ws_bytes, B, T, H, d_c, d_rope, page, pages, width, window,
                                     sinks, scale, io, cache, flags, None)


@pytest.mark.parametrize("kw, want", COMMON + [(dict(window=0), E_SHAPE), (dict(sinks=-1), E_SHAPE)])
def test_window_refusals(L, kw, want):
    assert window(L, **kw) == want


def prefill(L, qn=P, qr=P, UK=P, UV=P, kv=P, table=P, lens=P, out=P, lse=None, ws=P, ws_bytes=BIG, B=2, T=100, H=8, d_head=128, d_c=512, d_rope=64,
            page=64, pages=200, width=100, window=500, sinks=4, scale=0.1, io=BF16, cache=BF16):
    return L.mla_prefill_window(qn, qr, UK, UV, kv, table, lens, out, lse, ws, ws_bytes, B, T, H, d_head, d_c, d_rope, page, pages, width, window,
                                sinks, scale, io, cache, None)


@pytest.mark.parametrize("kw, want", [
    (dict(qn=None), E_NULL), (dict(qr=None), E_NULL), (dict(UK=None), E_NULL), (dict(UV=None), E_NULL), (dict(kv=None), E_NULL),
    (dict(table=None), E_NULL), (dict(lens=None), E_NULL), (dict(out=None), E_NULL),
    (dict(B=0), E_SHAPE), (dict(T=0), E_SHAPE), (dict(H=0), E_SHAPE), (dict(window=0), E_SHAPE), (dict(sinks=-1), E_SHAPE), (dict(width=0), E_SHAPE),
    (dict(scale=math.nan), E_SHAPE), (dict(width=1 << 26), E_SHAPE),
    (dict(io=F32), E_UNSUP), (dict(cache=FP8), E_UNSUP), (dict(d_head=64), E_UNSUP), (dict(d_c=128), E_UNSUP), (dict(page=32), E_UNSUP),
    (dict(B=8192, H=8), E_UNSUP), (dict(ws=None), E_WS), (dict(ws_bytes=1000), E_WS), (dict(ws=P + 64), E_WS)])
def test_prefill_window_refusals(L, kw, want):
    assert prefill(L, **kw) == want


def move(L, kv=P, scale=None, table=P, src=P, dst=P, B=2, n=4, row=1152, page=64, pages=10, width=4):
    return L.mla_cache_move(kv, scale, table, src, dst, B, n, row, page, pages, width, None)


@pytest.mark.parametrize("kw, want", [
    (dict(kv=None), E_NULL), (dict(table=None), E_NULL), (dict(src=None), E_NULL), (dict(dst=None), E_NULL), (dict(B=0), E_SHAPE),
    (dict(n=0), E_SHAPE), (dict(row=0), E_SHAPE), (dict(page=0), E_SHAPE), (dict(pages=-1), E_SHAPE), (dict(width=0), E_SHAPE),
    (dict(width=1 << 26), E_SHAPE), (dict(n=65), E_UNSUP), (dict(B=65536), E_UNSUP), (dict(row=4097), E_UNSUP)])
def test_move_refusals(L, kw, want):
    assert move(L, **kw) == want


def test_store_at_refusals(L):
    args = lambda slots=P, pos=P: (P, pos, slots, P, None, P, None, P, 1, 4, 512, 64, 576, 64, 10, 4, 1.0, 0, 1e-6, BF16, 9, None)
    assert L.mla_cache_store_at(*args(slots=None)) == E_NULL and L.mla_cache_store_at(*args(pos=None)) == E_NULL
    assert L.mla_cache_store_at(*args()) == E_UNSUP


def test_workspaces(L):
    t, w = L.mla_decode_tree_workspace_bytes, L.mla_decode_window_workspace_bytes
    assert t(64, 63, 28, 256, 4160) == 0                         # the query rows alone fill the chip: no partial results
    for B, T, H, rows in ((1, 1, 32, 64), (1, 8, 32, 1024), (4, 31, 32, 131104), (16, 1, 32, 8192)):
        n = t(B, T, H, 512, rows)
        assert n % 256 == 0 and n <= B * T * H * 64 * (512 + 1) * 4 + 512
        assert w(B, T, H, 512, rows, 1 << 30, 0) == n            # a window past the table is no window
    assert w(1, 1, 32, 512, 1 << 20, 64, 4) == w(1, 1, 32, 512, 1 << 24, 64, 4)
    for bad in ((0, 1, 1, 8, 1), (1, 0, 1, 8, 1), (1, 1, 0, 8, 1), (1, 1, 1, 0, 1), (1, 1, 1, 8, 0), (1, 65, 1, 8, 9), (1, 64, 129, 8, 9)):
        assert t(*bad) == 0
    assert w(1, 1, 32, 512, 64, 0, 0) == 0 and w(1, 1, 32, 512, 64, 1, -1) == 0
    p = L.mla_prefill_window_workspace_bytes
    assert p(1, 100, 8, 512, 1000, 128, 4) < p(1, 100, 8, 512, 1000, 4096, 4) < p(1, 100, 8, 512, 1000, 1 << 30, 4) == p(1, 100, 8, 512, 1000, 64000, 0)
    assert p(1, 100, 8, 512, 1000, 0, 4) == 0 and p(0, 100, 8, 512, 1000, 5, 4) == 0


def test_binding_refusals():
    q, qr = torch.zeros(1, 4, 8, 256, dtype=torch.bfloat16), torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16)
    kv, table, lens = torch.zeros(2, 64, 320, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    mask = torch.zeros(1, 4, dtype=torch.int64)
    bad = lambda e, f, *a, **k: pytest.raises(e, f, *a, **k)
    bad(ValueError, mla.decode_paged_tree, q, qr, kv, table, lens, mask[:, :3], 0.1)
    bad(TypeError, mla.decode_paged_tree, q, qr, kv, table, lens, mask.int(), 0.1)
    bad(TypeError, mla.decode_paged_tree, q, qr, kv, table, lens.long(), mask, 0.1)
    bad(ValueError, mla.decode_paged_tree, q, qr[:, :2], kv, table, lens, mask, 0.1)
    bad(ValueError, mla.decode_paged_tree, q[0], qr, kv, table, lens, mask, 0.1)
    bad(ValueError, mla.decode_paged_tree, q, qr, kv, table, lens, mask, 0.1, out=torch.zeros(1, 4, 8, 256))
    bad(ValueError, mla.decode_paged_tree, q, qr, kv, table, lens, mask, 0.1, lse=torch.zeros(1, 4, 7))
    bad(ValueError, mla.decode_paged_tree, q, qr, kv, table, lens, mask, 0.1)                       # not on the GPU
    bad(ValueError, mla.decode_paged_window, q, qr, kv, table.repeat(2, 1), lens, 5, 1, 0.1)
    bad(ValueError, mla.decode_paged_window, q, qr, kv, table, lens, 5, 1, 0.1, kv_scale=torch.zeros(2, 63))
    UK, UV = torch.zeros(8, 128, 256, dtype=torch.bfloat16), torch.zeros(8, 256, 128, dtype=torch.bfloat16)
    qn = torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16)
    bad(ValueError, mla.prefill_window, qn, qr, UK, UV.float(), kv, table, lens, 5, 1, 0.1)
    bad(ValueError, mla.prefill_window, qn, qr, UK, UV, kv, table, lens, 5, 1, 0.1, out=torch.zeros(1, 4, 8, 127, dtype=torch.bfloat16))
    src = torch.zeros(1, 3, dtype=torch.int32)
    bad(TypeError, layer.cache_move, kv, table, src.long(), src)
    bad(ValueError, layer.cache_move, kv, table, src, src[:, :2])
    bad(ValueError, layer.cache_move, kv, table, src, src, torch.zeros(2, 64))
    bad(ValueError, layer.cache_move, kv.to(torch.float8_e4m3fn), table, src, src)
    bad(ValueError, layer.cache_move, kv, table, src, src)                                          # not on the GPU


def test_windows_past_32_bits_are_wide_ones():
    wide = mla.decode_window_workspace_bytes(4, 1, 32, 512, 8192, 2 ** 31 - 1, 0)
    for big in (2 ** 31, 2 ** 32 + 64, 2 ** 40):
        assert mla.decode_window_workspace_bytes(4, 1, 32, 512, 8192, big, 0) == wide
        assert mla.decode_window_workspace_bytes(4, 1, 32, 512, 8192, 64, big) == wide
        assert mla.prefill_window_workspace_bytes(1, 100, 8, 512, 1000, big, big) == mla.prefill_window_workspace_bytes(1, 100, 8, 512, 1000, 64000, 64000)
        assert mla.decode_window_workspace_bytes(4, 1, 32, 512, 8192, -big, 0) == 0


def test_workspaces_are_those_of_the_kernels_that_are_used(L):
    """64 sequences of 63 x 32 query rows fill the chip: no kernel that such a call takes has partial results.  No call's partial results take more than 640 MB."""
    t, w = L.mla_decode_tree_workspace_bytes, L.mla_decode_window_workspace_bytes
    assert t(64, 63, 32, 512, 131136) == 0 and w(64, 63, 32, 512, 131136, 1 << 30, 0) == 0
    for B, T, H, d_c, rows in ((33, 64, 64, 512, 131136), (17, 63, 32, 512, 131136), (15, 64, 128, 512, 1 << 20), (100, 10, 100, 512, 70000), (40, 64, 64, 256, 1 << 18),
                               (9, 64, 128, 504, 1 << 20), (3000, 1, 1, 512, 1 << 20), (2, 64, 128, 512, 1 << 30)):
        assert max(t(B, T, H, d_c, rows), w(B, T, H, d_c, rows, 1 << 30, 4)) <= (640 << 20) + 512          # (two parts, each whole 256 bytes)


def test_workspaces_of_sizes_that_no_call_has(L):
    """Products past 64 bits: a size, whatever it is, and no arithmetic exception."""
    big = 2 ** 31 - 1
    for B, T, H, d_c, rows in ((1 << 20, 1, 8192, big, big), (big, 1, 1, big, big), (big, 64, 128, big, 1), (1, 1, 1, big, big), (65536, 1, 8192, big, 1 << 30)):
        assert L.mla_decode_tree_workspace_bytes(B, T, H, d_c, rows) <= (640 << 20) + 512
        assert L.mla_decode_window_workspace_bytes(B, T, H, d_c, rows, big, big) <= (640 << 20) + 512
