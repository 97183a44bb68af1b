"""Drafted trees, sliding windows with sinks and prompts under them against 64 bits (bounds: masked_reference.py); rows of the
cache moved; all of them together as a serving loop uses them."""
import math
import random

import pytest
import torch

from masked_reference import H as HALF, U, attend, close, gather
from paper_2502_07864_amd import layer, mla
from paper_2502_07864_amd.attention_layer import AttentionLayer

pytestmark = pytest.mark.gpu

DEV, BF, FP8, F32 = "cuda:0", torch.bfloat16, torch.float8_e4m3fn, torch.float32
SCALE = 192 ** -0.5
KINDS = {"bf16": (BF, BF), "fp8": (BF, FP8), "f32": (F32, F32), "f32_bf16": (F32, BF), "f32_fp8": (F32, FP8)}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


class Cache:
    """Sequences of `lens` rows on pages in random order; what lies on the pages' other rows, and on one spare page, is NaN."""

    def __init__(self, lens, d_c, d_rope, page, cache, seed=0, room=0):
        g, self.lens, self.page, self.d_c = gen(seed), lens, page, d_c
        width = max(1, -(-(max(lens) + room) // page))
        n = [-(-l // page) for l in lens]
        order = torch.randperm(sum(n) + 1, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
        row = d_c + d_rope
        self.kv = torch.full((sum(n) + 1, page, row), math.nan, device=DEV).to(cache)
        self.scale = torch.full((sum(n) + 1, page), math.nan, device=DEV) if cache == FP8 else None
        at = 0
        for b, l in enumerate(lens):
            self.table[b, :n[b]] = order[at:at + n[b]]
            at += n[b]
            self.put(b, range(l), torch.randn((l, row), generator=g, device=DEV))

    def places(self, b, rows):
        rows = torch.as_tensor(list(rows), device=DEV, dtype=torch.long)
        return self.table[b].long()[rows // self.page] * self.page + rows % self.page

    def put(self, b, rows, x):
        at, flat = self.places(b, rows), self.kv.view(-1, self.kv.shape[2])
        if self.scale is not None:
            s = x.abs().amax(1) / 448
            self.scale.view(-1)[at] = s
            flat.view(torch.uint8)[at] = (x / s[:, None]).to(FP8).view(torch.uint8)
        else:
            flat[at] = x.to(self.kv.dtype)

    def rows(self, n):
        x, there = gather(self.kv, self.scale, self.table, n)
        return x, there


def queries(B, T, H, d_c, d_rope, io, seed=1):
    g = gen(seed)
    q = torch.randn((B, T, H, d_c), generator=g, device=DEV) * (128 / max(d_c, 128)) ** 0.5
    return q.to(io), torch.randn((B, T, H, d_rope), generator=g, device=DEV).to(io) if d_rope else None


def tree_of(T, seed, width=4):
    rng, rows = random.Random(seed), []
    for i in range(T):
        up = rng.randint(max(-1, i - width), i - 1) if i else -1
        rows.append((rows[up] if up >= 0 else 0) | 1 << i)
    return rows


def signed(v):
    return v - (1 << 64) if v >> 63 else v


def check(c, q, qr, sees, call, io, scale=SCALE):
    """sees [B][T, n] of truth values.  The call's results against the definition."""
    B, T, H, d_c = q.shape
    n = sees.shape[2]
    x, there = c.rows(n)
    x = torch.where(there[..., None], x, torch.zeros_like(x))
    out, lse = call()
    assert out.dtype == io and out.shape == q.shape and lse.shape == (B, T, H)
    full = q.double() if qr is None else torch.cat((q.double(), qr.double()), -1)
    for b in range(B):
        o, l, eo, el = attend(full[b], x[b], x[b, :, :d_c], sees[b] & there[b], scale, io == BF)
        close(lse[b], l, el, f"lse of sequence {b}")
        close(out[b], o, eo, f"o of sequence {b}")
    return out, lse


def tree_sees(prefix, masks, T, n):
    s = torch.zeros((len(prefix), T, n), dtype=torch.bool)
    for b, p in enumerate(prefix):
        s[b, :, :p] = True
        for i in range(T):
            for k in range(T):
                if masks[b][i] >> k & 1 and p + k < n:
                    s[b, i, p + k] = True
    return s.to(DEV)


def run_tree(kind, prefix, T, H, d_c=512, d_rope=64, page=64, masks=None, seed=0, scale=SCALE, flags=0, poison=True, q=None):
    io, cache = KINDS[kind]
    c = Cache([p + T for p in prefix], d_c, d_rope, page, cache, seed)
    masks = masks or [tree_of(T, seed + b) for b in range(len(prefix))]
    if poison:                     # drafted rows that nobody sees
        for b, p in enumerate(prefix):
            unseen = [p + k for k in range(T) if not any(m >> k & 1 for m in masks[b])]
            if unseen:
                at = c.places(b, unseen)
                (c.kv.view(torch.uint8) if cache == FP8 else c.kv).view(-1, d_c + d_rope)[at] = 127 if cache == FP8 else math.nan
    q, qr = q or queries(len(prefix), T, H, d_c, d_rope, io, seed + 1)
    mask = torch.tensor([[signed(v) for v in m] for m in masks], dtype=torch.int64, device=DEV)
    lens = torch.tensor(prefix, dtype=torch.int32, device=DEV)
    call = lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, scale, kv_scale=c.scale, return_lse=True, flags=flags)
    return check(c, q, qr, tree_sees(prefix, masks, T, max(prefix) + T), call, io, scale), c, (q, qr), mask, lens


@pytest.mark.parametrize("flags", [0, mla.FLAG_PORTABLE_KERNEL])
@pytest.mark.parametrize("kind, d_c", [("bf16", 512), ("bf16", 256), ("fp8", 512), ("fp8", 256)])
@pytest.mark.parametrize("T, H", [(1, 1), (1, 32), (2, 32), (3, 28), (5, 16), (8, 32), (31, 7), (63, 28), (64, 3)])
def test_tree(kind, d_c, T, H, flags):
    run_tree(kind, [0, 1, 31, 32, 33, 65, 200], T, H, d_c, flags=flags)


@pytest.mark.parametrize("kind", ["f32", "f32_bf16", "f32_fp8"])
@pytest.mark.parametrize("d_c, d_rope, page", [(512, 64, 64), (256, 0, 7), (8, 8, 1), (392, 56, 24)])
def test_tree_portable_widths(kind, d_c, d_rope, page):
    run_tree(kind, [0, 5, 130], 6, 5, d_c, d_rope, page)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("page", [1, 16, 24, 32, 96, 128])
def test_tree_pages(kind, page):
    run_tree(kind, [3, 127, 160, 300], 9, 32, page=page)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("prefix, T, H", [([3000], 4, 32), ([1500, 2], 16, 32), ([900] * 3, 40, 40), ([5000, 0, 4000, 17], 2, 64)])
def test_tree_long(kind, prefix, T, H):
    run_tree(kind, prefix, T, H, 512)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_masks(kind):
    """Rows that see nothing, everything, only others, and bits past the drafted tokens."""
    T = 40
    every = (1 << 64) - 1
    masks = [[0] * T, [every] * T, [1 << (i * 7 + 3) % T for i in range(T)], [every << T & every] * T, [(1 << i) - 1 for i in range(T)]]
    for prefix in ([0] * 5, [64, 32, 1, 0, 500]):
        (out, lse), *_ = run_tree(kind, prefix, T, 8, masks=masks)
        if prefix[0] == 0:
            assert (out[0] == 0).all() and torch.isneginf(lse[0]).all() and (out[3] == 0).all() and (out[4, 0] == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_chain_is_multi(kind):
    """A lower triangle is decode_paged_multi's mask; one tree for all sequences."""
    T, H = 4, 32
    (out, lse), c, (q, qr), _, lens = run_tree(kind, [100, 333, 64], T, H, masks=[[(2 << i) - 1 for i in range(T)]] * 3)
    one = torch.tensor([(2 << i) - 1 for i in range(T)], dtype=torch.int64, device=DEV)
    again, _ = mla.decode_paged_tree(q, qr, c.kv, c.table, lens, one, SCALE, kv_scale=c.scale, return_lse=True)
    assert torch.equal(again, out)
    multi, lse2 = mla.decode_paged_multi(q, qr, c.kv, c.table, lens + T, SCALE, kv_scale=c.scale, return_lse=True)
    assert (multi.double() - out.double()).abs().max() <= 0.02 * out.double().abs().max()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_tree_other_branches_do_not_leak(kind, what):
    """A drafted row that is not finite: whoever does not see it gets the same bits as beside a finite one."""
    T, H, prefix = 20, 28, [70, 45]
    masks = [tree_of(T, b) for b in range(2)]
    (out, lse), c, (q, qr), mask, lens = run_tree(kind, prefix, T, H, masks=masks)
    for bad in (0, 7, 19):
        for b in range(2):
            row, s = c.kv.view(-1, 576), c.scale
            at = c.places(b, [prefix[b] + bad])
            if kind == "fp8":
                kept = s.view(-1)[at].clone()
                s.view(-1)[at] = math.nan if what == "nan" else math.inf
            else:
                kept = row[at].clone()
                row[at] = math.nan if what == "nan" else math.inf
            got, l2 = mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=s, return_lse=True)
            for i in range(T):
                if masks[b][i] >> bad & 1:
                    assert not torch.isfinite(got[b, i].float()).any()
                else:
                    assert torch.equal(got[b, i], out[b, i]) and torch.equal(l2[b, i], lse[b, i]), (b, bad, i)
            assert torch.equal(got[1 - b], out[1 - b])
            if kind == "fp8":
                s.view(-1)[at] = kept
            else:
                row[at] = kept


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_pages_that_are_not_there(kind):
    T, H = 10, 32
    for drop in ([(0, 0)], [(0, 2), (1, 1)], [(0, 3), (1, 0), (1, 1)]):
        io, cache = KINDS[kind]
        c = Cache([200 + T, 90 + T], 512, 64, 64, cache, 3)
        for b, p in drop:
            c.table[b, p] = (-1, c.kv.shape[0], 1 << 30)[(b + p) % 3]
        masks = [tree_of(T, 5), tree_of(T, 6)]
        q, qr = queries(2, T, H, 512, 64, io)
        mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
        lens = torch.tensor([200, 90], dtype=torch.int32, device=DEV)
        check(c, q, qr, tree_sees([200, 90], masks, T, 210),
              lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True), io)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_past_the_table_and_odd_lengths(kind):
    """Drafted rows behind the table's end are not there; lengths below zero and past the table are its ends."""
    T, H = 12, 16
    io, cache = KINDS[kind]
    c = Cache([128, 128, 128], 512, 64, 64, cache, 4)
    masks = [[(2 << i) - 1 for i in range(T)]] * 3
    q, qr = queries(3, T, H, 512, 64, io)
    mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
    lens = torch.tensor([120, -5, 4000], dtype=torch.int32, device=DEV)
    check(c, q, qr, tree_sees([120, 0, 128], masks, T, 128),
          lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True), io)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("scale", [-SCALE, 0.0, 3.0])
def test_tree_scales(kind, scale):
    run_tree(kind, [40, 600], 7, 20, scale=scale)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("where", [0, 40, 700, 1495])
def test_tree_score_that_dominates(kind, where):
    """One row whose score is far above those before it (the running reference moves)."""
    io, cache = KINDS[kind]
    T, H, P = 6, 32, 1490
    c = Cache([P + T], 512, 64, 64, cache, 8)
    q, qr = queries(1, T, H, 512, 64, io)
    big = torch.cat((q[0, 2, 5], qr[0, 2, 5])).float() * 12.0
    c.put(0, [where], big[None])
    masks = [tree_of(T, 2)]
    masks[0][2] |= 1 << 5
    mask = torch.tensor(masks, dtype=torch.int64, device=DEV)
    lens = torch.tensor([P], dtype=torch.int32, device=DEV)
    check(c, q, qr, tree_sees([P], masks, T, P + T),
          lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True), io)


# ------------------------------------------------------------------ windows

def window_sees(lens, T, window, sinks, n):
    j = torch.arange(n)
    s = torch.zeros((len(lens), T, n), dtype=torch.bool)
    for b, l in enumerate(lens):
        for i in range(T):
            t = l - T + i
            if t >= 0:
                s[b, i] = (j <= t) & ((j > t - window) | (j < sinks))
    return s.to(DEV)


def give_back(c, sees):
    """Pages of which no token sees a row go; so do the rows of the others that nobody sees."""
    for b, l in enumerate(c.lens):
        seen = sees[b].any(0)
        for p in range(-(-l // c.page)):
            rows = [j for j in range(p * c.page, min(l, (p + 1) * c.page))]
            if not seen[rows].any():
                c.table[b, p] = -1
        dead = [j for j in range(l) if not seen[j] and c.table[b, j // c.page] >= 0]
        if dead:
            at = c.places(b, dead)
            if c.scale is not None:
                c.scale.view(-1)[at] = math.nan
            else:
                c.kv.view(-1, c.kv.shape[2])[at] = math.nan


def run_window(kind, lens, T, H, window, sinks, d_c=512, d_rope=64, page=64, seed=0, flags=0, scale=SCALE):
    io, cache = KINDS[kind]
    c = Cache(lens, d_c, d_rope, page, cache, seed)
    sees = window_sees(lens, T, window, sinks, max(lens))
    give_back(c, sees)
    q, qr = queries(len(lens), T, H, d_c, d_rope, io, seed + 1)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    call = lambda: mla.decode_paged_window(q, qr, c.kv, c.table, n, window, sinks, scale, kv_scale=c.scale, return_lse=True, flags=flags)
    return check(c, q, qr, sees, call, io, scale), c, (q, qr), n


@pytest.mark.parametrize("flags", [0, mla.FLAG_PORTABLE_KERNEL])
@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("T, H", [(1, 1), (1, 32), (2, 28), (4, 32), (7, 40)])
@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 4), (33, 1), (64, 64), (100, 100), (257, 4), (5000, 3)])
def test_window(kind, T, H, window, sinks, flags):
    run_window(kind, [1, 31, 64, 65, 130, 700, 1025], T, H, window, sinks, flags=flags)


@pytest.mark.parametrize("kind, d_c, d_rope, page", [("f32", 512, 64, 64), ("f32_bf16", 256, 64, 5), ("f32_fp8", 40, 8, 64), ("bf16", 256, 64, 64),
                                                     ("fp8", 256, 64, 128), ("bf16", 512, 64, 16), ("bf16", 128, 0, 32), ("bf16", 512, 64, 32)])
def test_window_widths(kind, d_c, d_rope, page):
    for window, sinks in ((50, 4), (200, 0)):
        run_window(kind, [3, 90, 400, 1111], 3, 12, window, sinks, d_c, d_rope, page)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("lens, T, H, window, sinks", [
    ([20000], 1, 32, 4096, 4), ([9000, 100, 6000], 1, 28, 1024, 128), ([3000] * 5, 40, 32, 600, 4), ([700], 100, 3, 64, 1), ([2500], 16, 64, 2147483647, 2147483647)])
def test_window_long(kind, lens, T, H, window, sinks):
    run_window(kind, lens, T, H, window, sinks)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_window_wide_open_is_multi(kind):
    (out, lse), c, (q, qr), n = run_window(kind, [64, 300, 1000], 2, 32, 5000, 0)
    multi = mla.decode_paged_multi(q, qr, c.kv, c.table, n, SCALE, kv_scale=c.scale)
    assert (multi.double() - out.double()).abs().max() <= 0.02 * out.double().abs().max()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_window_other_tokens_rows_do_not_leak(kind):
    """A row that only earlier, or only later tokens see."""
    T, H, L, window = 5, 32, 400, 100
    (out, lse), c, (q, qr), n = run_window(kind, [L], T, H, window, 4)
    for j in (L - T - window + 1, L - T - window + 3, L - 1, L - 3):
        at = c.places(0, [j])
        x = c.scale.view(-1) if kind == "fp8" else c.kv.view(-1, 576)
        kept = x[at].clone()
        for bad in (math.nan, math.inf):
            x[at] = bad
            got = mla.decode_paged_window(q, qr, c.kv, c.table, n, window, 4, SCALE, kv_scale=c.scale)
            for i in range(T):
                t = L - T + i
                if t - window < j <= t:
                    assert not torch.isfinite(got[0, i].float()).any()
                else:
                    assert torch.equal(got[0, i], out[0, i]), (j, i)
        x[at] = kept


# ------------------------------------------------------------------ prompts

def run_prefill(lens, T, H, window, sinks, d_c=512, seed=0, scale=SCALE, misaligned=False, call=mla.prefill_window):
    c = Cache(lens, d_c, 64, 64, BF, seed)
    sees = window_sees(lens, T, window, sinks, max(lens))
    give_back(c, sees)
    kv = c.kv
    if misaligned:
        kv = torch.empty(c.kv.numel() + 1, dtype=BF, device=DEV)[1:].view(c.kv.shape)
        kv.copy_(c.kv)
    g, B = gen(seed + 1), len(lens)
    qn, qr = (torch.randn((B, T, H, d), generator=g, device=DEV).to(BF) for d in (128, 64))
    UK, UV = ((torch.randn(s, generator=g, device=DEV) * d_c ** -0.5).to(BF) for s in ((H, 128, d_c), (H, d_c, 128)))
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse = call(qn, qr, UK, UV, kv, c.table, n, window, sinks, scale, return_lse=True)
    x, there = c.rows(max(lens))
    for b in range(B):
        live = sees[b].any(0) & there[b]
        xb = torch.where(live[:, None], x[b], torch.zeros_like(x[b]))
        lat, rope = xb[:, :d_c], xb[:, d_c:].expand(H, -1, -1)
        both = lat.expand(H, *lat.shape)
        k, v = torch.bmm(both, UK.double().transpose(1, 2).contiguous()), torch.bmm(both, UV.double())
        sums = (d_c + 8) * U
        dk = HALF * k.abs() + sums * torch.bmm(both.abs(), UK.double().abs().transpose(1, 2).contiguous())
        dv = HALF * v.abs() + sums * torch.bmm(both.abs(), UV.double().abs())
        o, l, eo, el = attend(torch.cat((qn[b], qr[b]), -1).double(), torch.cat((k, rope), -1), v, sees[b] & there[b], scale, True,
                              torch.cat((dk, torch.zeros_like(rope)), -1), dv)
        # (the normaliser sums rounded weights here: half a step of bf16 more on the lse)
        close(lse[b], l, el + HALF * (~torch.isneginf(l)), f"lse of sequence {b}")
        close(out[b], o, eo, f"out of sequence {b}")
    return out, lse, (qn, qr, UK, UV), c, n


@pytest.mark.parametrize("d_c", [256, 512])
@pytest.mark.parametrize("lens, T, H, window, sinks", [
    ([1], 1, 1, 1, 0), ([33, 64, 65], 33, 2, 20, 4), ([200, 129], 129, 3, 64, 0), ([300, 301], 300, 2, 1, 1), ([500], 500, 4, 96, 70),
    ([1000, 260], 250, 2, 130, 4), ([2000], 137, 3, 500, 4), ([2000, 700, 1500], 64, 2, 31, 200), ([400], 400, 2, 100000, 3), ([100, 40], 60, 2, 30, 4),
    ([4500], 130, 2, 4200, 300)])
def test_prefill_window(d_c, lens, T, H, window, sinks):
    run_prefill(lens, T, H, window, sinks, d_c)


def test_prefill_window_misaligned_cache():
    run_prefill([500, 90], 80, 2, 100, 4, 256, misaligned=True)


@pytest.mark.parametrize("scale", [-SCALE, 0.0])
def test_prefill_window_scales(scale):
    run_prefill([300], 200, 2, 90, 4, 256, scale=scale)


def causal(qn, qr, UK, UV, kv, table, n, window, sinks, scale, return_lse):
    return mla.prefill_mha(qn, qr, UK, UV, kv, table, n, scale, return_lse=True)


def test_prefill_window_wide_open_is_causal():
    """Both calls are as near to the same reference as the count of roundings says (a few workgroups' keys are cut into chunks, so
    that the weights are rounded against other maxima)."""
    for call in (mla.prefill_window, causal):
        run_prefill([700, 300], 300, 4, 2147483647, 0, call=call)


def test_prefill_window_wide_open_has_the_bits_of_causal_where_nothing_is_cut():
    g, c = gen(5), Cache([700, 600], 256, 64, 64, BF, 4)
    qn, qr = (torch.randn((2, 600, 64, d), generator=g, device=DEV).to(BF) for d in (128, 64))
    UK, UV = ((torch.randn(s, generator=g, device=DEV) / 16).to(BF) for s in ((64, 128, 256), (64, 256, 128)))
    n = torch.tensor([700, 600], dtype=torch.int32, device=DEV)
    out, lse = mla.prefill_window(qn, qr, UK, UV, c.kv, c.table, n, 2147483647, 0, SCALE, return_lse=True)
    ref, l2 = causal(qn, qr, UK, UV, c.kv, c.table, n, 0, 0, SCALE, True)
    assert torch.equal(out, ref) and torch.equal(lse, l2)


@pytest.mark.parametrize("lens, T, H, window, sinks", [([9000], 1, 2, 7000, 4), ([9000, 40, 5000], 3, 3, 9000, 700), ([6000], 129, 1, 5000, 0)])
def test_prefill_window_in_chunks(lens, T, H, window, sinks):
    run_prefill(lens, T, H, window, sinks, 256)


@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_prefill_window_rows_do_not_leak(what):
    """A row that is not finite reaches exactly the tokens that see it."""
    T, L, window, sinks = 300, 520, 90, 4
    out, _, (qn, qr, UK, UV), c, n = run_prefill([L], T, 2, window, sinks, 256)
    for j in (3, L - T - window + 5, L - T + 100, L - 1):
        at = c.places(0, [j])
        kept = c.kv.view(-1, 320)[at].clone()
        c.kv.view(-1, 320)[at] = what
        got = mla.prefill_window(qn, qr, UK, UV, c.kv, c.table, n, window, sinks, SCALE)
        sees = window_sees([L], T, window, sinks, L)[0][:, j]
        assert torch.equal(got[0, ~sees], out[0, ~sees]), j
        assert not torch.isfinite(got[0, sees].float()).any(), j
        c.kv.view(-1, 320)[at] = kept


def test_prefill_window_missing_pages():
    T, L = 100, 400
    c = Cache([L], 256, 64, 64, BF, 2)
    c.table[0, 4] = -1
    g = gen(1)
    qn, qr = (torch.randn((1, T, 2, d), generator=g, device=DEV).to(BF) for d in (128, 64))
    UK, UV = ((torch.randn(s, generator=g, device=DEV) / 16).to(BF) for s in ((2, 128, 256), (2, 256, 128)))
    n = torch.tensor([L], dtype=torch.int32, device=DEV)
    out = mla.prefill_window(qn, qr, UK, UV, c.kv, c.table, n, 150, 4, SCALE)
    x, there = c.rows(L)
    x = torch.where(there[..., None], x, torch.zeros_like(x))[0]
    lat = x[:, :256].expand(2, -1, -1)
    k = torch.cat((torch.bmm(lat, UK.double().transpose(1, 2).contiguous()), x[:, 256:].expand(2, -1, -1)), -1)
    v = torch.bmm(lat, UV.double())
    o, *_ = attend(torch.cat((qn[0], qr[0]), -1).double(), k, v, window_sees([L], T, 150, 4, L)[0] & there[0], SCALE, True)
    assert (out[0].double() - o).abs().max() <= 0.03 * o.abs().max()


# ------------------------------------------------------------------ streams, graphs, workspaces

def test_calls_in_a_graph():
    """Captured once and replayed on changing inputs and lengths, with eager calls between the replays; two graphs share a workspace."""
    T, H = 6, 32
    _, c, (q, qr), mask, lens = run_tree("bf16", [1500, 40], T, H)
    n = lens + T
    ws = torch.full((max(mla.decode_tree_workspace_bytes(2, T, H, 512, c.table.shape[1] * 64),
                         mla.decode_window_workspace_bytes(2, T, H, 512, c.table.shape[1] * 64, 300, 4)),), 255, dtype=torch.uint8, device=DEV)
    out, out2 = torch.empty_like(q), torch.empty_like(q)
    tree = lambda o: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, workspace=ws, out=o)
    window = lambda o: mla.decode_paged_window(q, qr, c.kv, c.table, n, 300, 4, SCALE, workspace=ws, out=o)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        tree(out), window(out2)
    torch.cuda.current_stream().wait_stream(s)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        tree(out)
    with torch.cuda.graph(graphs[1]):
        window(out2)
    for step in range(4):
        q.copy_(queries(2, T, H, 512, 64, BF, 50 + step)[0])
        lens.copy_(torch.tensor([1500 - 97 * step, 40 + step], dtype=torch.int32))
        n.copy_(lens + T)
        for g in graphs:
            g.replay()
        a, b = tree(torch.empty_like(q)), window(torch.empty_like(q))
        torch.cuda.synchronize()
        # (bits: the second sequence grows over rows that hold NaN)
        assert torch.equal(a.view(torch.int16), out.view(torch.int16)) and torch.equal(b.view(torch.int16), out2.view(torch.int16)), step


def test_same_bits_every_time():
    for kind in ("bf16", "fp8"):
        (out, lse), c, (q, qr), mask, lens = run_tree(kind, [2000, 700, 5], 16, 32)
        for _ in range(5):
            o, l = mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True)
            assert torch.equal(o, out) and torch.equal(l, lse)


# ------------------------------------------------------------------ moves

@pytest.mark.parametrize("cache, row", [(BF, 576), (FP8, 576), (F32, 320), (BF, 33), (FP8, 13), (BF, 70), (F32, 1)])
@pytest.mark.parametrize("B, n, page", [(1, 1, 64), (3, 5, 64), (2, 64, 16), (7, 33, 3)])
def test_move(cache, row, B, n, page):
    g, rng = gen(n + row), random.Random(n)
    width = -(-300 // page)
    table = torch.randperm(B * width + 2, generator=g, device=DEV)[:B * width].view(B, width).to(torch.int32)
    raw = torch.randint(0, 256, (B * width + 2, page, row * torch.empty((), dtype=cache).element_size()), generator=g, device=DEV, dtype=torch.uint8)
    kv, scale = raw.view(cache), torch.rand((B * width + 2, page), generator=g, device=DEV) if cache == FP8 else None
    table[0, 1] = -1
    src, dst = [], []
    for b in range(B):                  # chains, swaps and rows that stay: sources and destinations overlap
        places = rng.sample(range(300), n)
        to = places[1:] + places[:1] if b % 2 == 0 else rng.sample(range(300), n)
        for lst in (places, to):
            for k in range(0, n, 9):
                if n > 1:
                    lst[k] = (-1, 300 + 2 * page, 1 << 30)[k % 3]
        src.append(places)
        dst.append(to)
    want, want_scale = raw.clone().cpu(), None if scale is None else scale.clone().cpu()
    t, before, before_scale = table.cpu(), raw.cpu().clone(), None if scale is None else scale.cpu().clone()
    def place(b, j):
        if j < 0 or j >= width * page or t[b, j // page] < 0:
            return None
        return int(t[b, j // page]), j % page
    for b in range(B):
        for i, j in zip(src[b], dst[b]):
            p, q = place(b, i), place(b, j)
            if p and q:
                want[q] = before[p]
                if scale is not None:
                    want_scale[q] = before_scale[p]
    layer.cache_move(kv, table, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (src, dst)), kv_scale=scale)
    assert torch.equal(raw.cpu(), want) and (scale is None or torch.equal(scale.cpu(), want_scale))


def test_move_off_sixteen_bytes():
    raw = torch.arange(4 * 64 * 20 + 2, device=DEV).to(torch.uint8)[2:].view(4, 64, 20)
    kv, table = raw.view(BF), torch.tensor([[2, 0]], dtype=torch.int32, device=DEV)
    want = raw.clone()
    want[2, 5], want[0, 1] = raw[0, 9], raw[2, 5]
    layer.cache_move(kv, table, torch.tensor([[73, 5]], dtype=torch.int32, device=DEV), torch.tensor([[5, 65]], dtype=torch.int32, device=DEV))
    assert torch.equal(raw, want)


@pytest.mark.parametrize("layout", [layer.ROPE_INTERLEAVED, layer.ROPE_HALF])
@pytest.mark.parametrize("cache", [BF, FP8])
@pytest.mark.parametrize("row", [576, 64 + 6])
def test_store_at_slots(layout, cache, row):
    """A row stored elsewhere is the row stored at its position, moved."""
    d_rope = 64 if row == 576 else 6
    B, T = 2, 5
    g = gen(row)
    rows = torch.randn((B, T, row), generator=g, device=DEV)
    freq, gain = layer.rope_frequencies(d_rope)
    table = torch.tensor([[3, 1], [0, 2]], dtype=torch.int32, device=DEV)
    new = lambda: (torch.zeros((4, 64, row), device=DEV).to(cache), torch.zeros((4, 64), device=DEV) if cache == FP8 else None)
    pos = torch.tensor([[7, 8, 8, 9, 70], [1, 2, 2, 2, 3]], dtype=torch.int32, device=DEV)
    slots = torch.tensor([[10, 11, 12, 13, 100], [64, 65, 66, -1, 128]], dtype=torch.int32, device=DEV)
    (a, sa), _ = new(), None
    layer.cache_store(rows, pos, freq, a, table, row - d_rope, gain, layout, kv_scale=sa, slots=slots)
    seen = torch.zeros((4, 64), dtype=torch.bool, device=DEV)
    for b in range(B):
        for i in range(T):
            p, s = int(pos[b, i]), int(slots[b, i])
            if not 0 <= s < 128:
                continue
            one, s1 = new()
            layer.cache_store(rows[b:b + 1, i:i + 1], pos[b:b + 1, i:i + 1].contiguous(), freq, one, table[b:b + 1], row - d_rope, gain, layout,
                              kv_scale=s1)
            at, to = (int(table[b, p // 64]), p % 64), (int(table[b, s // 64]), s % 64)
            assert torch.equal(a[to].view(torch.uint8), one[at].view(torch.uint8)) and (sa is None or sa[to] == s1[at])
            seen[to] = True
    assert (a.view(torch.uint8)[~seen] == 0).all()


# ------------------------------------------------------------------ together

def make_layer(H=16, D=1024, d_c=256, **kw):
    g = gen(9)
    w = lambda *s: torch.randn(s, generator=g, device=DEV) * s[-1] ** -0.5
    return AttentionLayer(w(H * 192, D), w(d_c + 64, D), w(H, 128, d_c).to(BF), (torch.randn((H, d_c, 128), generator=g, device=DEV) * d_c ** -0.5).to(BF),
                          w(D, H * 128), torch.ones(D, dtype=BF, device=DEV), layer.rope_frequencies(64), SCALE, **kw)


@pytest.mark.parametrize("cache", [BF, FP8])
def test_drafted_tree_through_the_layer(cache):
    """A tree verified, its accepted path moved, the next tokens decoded: the same as these tokens decoded one at a time."""
    lay, D, prefix, T = make_layer(), 1024, [100, 61], 12
    g = gen(3)
    new = lambda: (torch.zeros((8, 64, 320), device=DEV).to(cache), torch.zeros((8, 64), device=DEV) if cache == FP8 else None)
    table = torch.tensor([[5, 2, 7], [0, 3, 1]], dtype=torch.int32, device=DEV)
    (kv, ks), B = new(), 2
    lens = torch.tensor(prefix, dtype=torch.int32, device=DEV)
    for b in range(B):
        x = torch.randn((1, prefix[b], D), generator=g, device=DEV).to(BF)
        pos = torch.arange(prefix[b], dtype=torch.int32, device=DEV)[None]
        codes, scales, *_ = layer.rms_norm_fp8(x[0], lay.norm_weight, lay.eps)
        layer.cache_store(layer.gemm_fp8(codes, scales, *lay.W_DKVR, dtype=F32)[None], pos, lay.freq, kv, table[b:b + 1], 256, kv_scale=ks)
    masks = [tree_of(T, 20 + b) for b in range(B)]
    depth = [[bin(m).count("1") - 1 for m in r] for r in masks]
    drafted = torch.randn((B, T, D), generator=g, device=DEV).to(BF)
    positions = torch.tensor([[p + d for d in r] for p, r in zip(prefix, depth)], dtype=torch.int32, device=DEV)
    slots = torch.tensor([[p + k for k in range(T)] for p in prefix], dtype=torch.int32, device=DEV)
    one_by_one, one_scale = kv.clone(), None if ks is None else ks.clone()
    out, _ = lay.decode_tree(drafted, positions, slots, kv, table, lens, torch.tensor(masks, dtype=torch.int64, device=DEV), kv_scale=ks)
    # the longest path of each tree
    paths = [[k for k in range(T) if r[max(range(T), key=lambda i: d[i])] >> k & 1] for r, d in zip(masks, depth)]
    n = max(len(p) for p in paths)
    src = torch.tensor([[p + k for k in path] + [-1] * (n - len(path)) for p, path in zip(prefix, paths)], dtype=torch.int32, device=DEV)
    dst = torch.tensor([[p + i for i in range(n)] for p in prefix], dtype=torch.int32, device=DEV)
    layer.cache_move(kv, table, src, dst, kv_scale=ks)
    for b in range(B):
        for i, k in enumerate(paths[b]):
            at = torch.tensor([[prefix[b] + i]], dtype=torch.int32, device=DEV)
            ref, _ = lay.decode(drafted[b:b + 1, k:k + 1], at, one_by_one, table[b:b + 1], at[0] + 1, kv_scale=one_scale)
            assert (ref[0, 0].double() - out[b, k].double()).norm() <= 2e-2 * ref.double().norm()
            page, row = int(table[b, (prefix[b] + i) // 64]), (prefix[b] + i) % 64
            assert torch.equal(kv[page, row].view(torch.uint8), one_by_one[page, row].view(torch.uint8))
    after = torch.randn((B, 1, D), generator=g, device=DEV).to(BF)
    ends = torch.tensor([p + len(path) for p, path in zip(prefix, paths)], dtype=torch.int32, device=DEV)
    a, _ = lay.decode(after, ends[:, None], kv, table, ends + 1, kv_scale=ks)
    r, _ = lay.decode(after, ends[:, None], one_by_one, table, ends + 1, kv_scale=one_scale)
    assert torch.equal(a, r)


def test_window_through_the_layer():
    """A prompt, then tokens one and two at a time, under a window: the same as a prompt of all of them; pages behind the window are
    given back on the way."""
    lay, D, L, new = make_layer(window=100, sinks=4), 1024, 300, 5
    x = torch.randn((1, L + new, D), generator=gen(2), device=DEV).to(BF)
    table = torch.tensor([[4, 1, 0, 5, 3]], dtype=torch.int32, device=DEV)
    kv, whole = (torch.zeros((6, 64, 320), dtype=BF, device=DEV) for _ in range(2))
    at = torch.arange(L + new, dtype=torch.int32, device=DEV)[None]
    n = lambda k: torch.tensor([k], dtype=torch.int32, device=DEV)
    ref, _ = lay.prefill(x, at, whole, table, n(L + new))
    got, _ = lay.prefill(x[:, :L], at[:, :L].contiguous(), kv, table, n(L))
    assert (got.double() - ref[:, :L].double()).norm() <= 1e-2 * ref.double().norm()
    kv[1], kv[0] = math.nan, math.nan          # rows 64 .. 191 are behind the window of row 300 and past the sinks
    table[0, 1] = table[0, 2] = -1
    for i, T in ((L, 1), (L + 1, 2), (L + 3, 1), (L + 4, 1)):
        got, _ = lay.decode(x[:, i:i + T].contiguous(), at[:, i:i + T].contiguous(), kv, table, n(i + T))
        assert (got.double() - ref[:, i:i + T].double()).norm() <= 2e-2 * ref[:, i:i + T].double().norm()
    with pytest.raises(ValueError):
        lay.decode_tree(x[:, :1], at[:, :1], at[:, :1], kv, table, n(1), torch.ones(1, dtype=torch.int64, device=DEV))
