"""Rows that are not finite, in tiles that every token of the call sees whole and in others (tests/test_gpu_masked.py has them in drafted
rows and at a window's edge): the tokens that see such a row are NaN, on every kernel and whichever tile it lies in; the others keep
their bits."""
import math

import pytest
import torch

from paper_2502_07864_amd import mla
from test_gpu_masked import BF, Cache, DEV, SCALE, gen, run_tree, run_window, window_sees
from test_gpu_masked_sizes import crowd

pytestmark = pytest.mark.gpu

# (committed rows, tokens, heads): the kernel for few query rows in one chunk and in several, the one for many rows in one chunk
CALLS = {"few": ([310], 8, 32), "few, in chunks": ([3000], 4, 32), "many": (crowd([310]), 20, 28)}


def tree_call(kind, which, flags=0, d_c=512):
    prefix, T, H = CALLS[which]
    (out, lse), c, (q, qr), mask, lens = run_tree(kind, prefix, T, H, d_c, flags=flags)
    b = max(range(len(prefix)), key=lambda i: prefix[i])
    call = lambda: mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True, flags=flags)
    return call, out, lse, c, (q, qr), b, prefix[b]


@pytest.mark.parametrize("which", CALLS)
@pytest.mark.parametrize("flags", [0, mla.FLAG_PORTABLE_KERNEL])
@pytest.mark.parametrize("kind, d_c", [("bf16", 512), ("bf16", 256), ("fp8", 512), ("fp8", 256), ("f32", 512)])
def test_an_infinite_score_in_the_middle_of_a_prefix(kind, d_c, flags, which):
    """One infinite value of a row (an infinite scale of an fp8 one): where the score is +inf nothing of the result is finite."""
    call, out, lse, c, (q, qr), b, n = tree_call(kind, which, flags, d_c)
    for j in (n // 2 + 15, n - 100):          # (no wavefront's first tile)
        at = c.places(b, [j])
        if kind == "fp8":
            rows = c.scale.view(-1)
            kept = rows[at].clone()
            rows[at] = math.inf
            up = torch.ones(out[b].shape[:2], dtype=torch.bool, device=DEV)      # (every value of the row is infinite or NaN, and so is what it is weighed into)
        else:
            rows = c.kv.view(-1, d_c + 64)
            kept = rows[at].clone()
            rows[at, 77] = math.inf
            up = q[b, :, :, 77] > 0
        got, l2 = call()
        assert not torch.isfinite(got[b][up].float()).any(), j
        others = torch.arange(len(out), device=DEV) != b
        assert torch.equal(got[others], out[others]) and torch.equal(l2[others], lse[others])
        rows[at] = kept
        got, l2 = call()
        assert torch.equal(got, out) and torch.equal(l2, lse)


def all_nan(x):
    return bool(torch.isnan(x.float()).all())


# one infinite value: of the latent part, whose score is +inf for some heads and -inf for others, or of the rope part, where the
# values themselves are finite
@pytest.mark.parametrize("column", [3, -9])
@pytest.mark.parametrize("which", CALLS)
@pytest.mark.parametrize("flags", [0, mla.FLAG_PORTABLE_KERNEL])
@pytest.mark.parametrize("kind, d_c", [("bf16", 512), ("bf16", 256), ("fp8", 512), ("f32", 512)])
def test_whoever_sees_an_infinite_row_is_nan_in_any_tile(kind, d_c, flags, which, column):
    call, out, lse, c, (q, qr), b, n = tree_call(kind, which, flags, d_c)
    # the first rows, whole tiles, the tile in which the prefix ends
    for j in (0, 5, n // 2, n - 70, n - 1):
        at = c.places(b, [j])
        rows = c.scale.view(-1) if kind == "fp8" else c.kv.view(-1, d_c + 64)[:, column]
        for what in (math.inf, -math.inf):
            kept = rows[at].clone()
            rows[at] = what
            got, l2 = call()
            assert all_nan(got[b]) and all_nan(l2[b]), (j, what)
            others = torch.arange(len(out), device=DEV) != b
            assert torch.equal(got[others], out[others]) and torch.equal(l2[others], lse[others])
            rows[at] = kept


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_an_infinite_drafted_row_makes_its_tokens_nan_whole(kind):
    T, H, prefix = 9, 28, [77, 640]
    masks = [[(2 << i) - 1 for i in range(T)]] * 2
    (out, lse), c, (q, qr), mask, lens = run_tree(kind, prefix, T, H, masks=masks)
    for b in range(2):
        for k in (0, 4, 8):
            at = c.places(b, [prefix[b] + k])
            rows = c.scale.view(-1) if kind == "fp8" else c.kv.view(-1, 576)[:, 3]
            kept = rows[at].clone()
            rows[at] = -math.inf
            got, l2 = mla.decode_paged_tree(q, qr, c.kv, c.table, lens, mask, SCALE, kv_scale=c.scale, return_lse=True)
            assert all_nan(got[b, k:]) and all_nan(l2[b, k:])
            assert torch.equal(got[b, :k], out[b, :k]) and torch.equal(l2[b, :k], lse[b, :k]) and torch.equal(got[1 - b], out[1 - b])
            rows[at] = kept


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_an_infinite_row_in_a_chunk_without_weight(kind):
    """A row that outweighs all others by more than fp32 holds lies in another chunk."""
    call, out, lse, c, (q, qr), b, n = tree_call(kind, "few, in chunks")
    c.put(0, [2900], torch.cat((q[0, 1, 5], qr[0, 1, 5])).float()[None] * 60.0)
    rows = c.scale.view(-1) if kind == "fp8" else c.kv.view(-1, 576)[:, 3]
    rows[c.places(0, [40])] = -math.inf
    got, l2 = call()
    assert all_nan(got) and all_nan(l2)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("lens, T, H", [([700], 3, 32), (crowd([700], 20), 20, 28)])
def test_an_infinite_row_under_a_window(kind, lens, T, H):
    window, sinks = 300, 40
    (out, lse), c, (q, qr), n = run_window(kind, lens, T, H, window, sinks)
    b = max(range(len(lens)), key=lambda i: lens[i])
    rows = c.scale.view(-1) if kind == "fp8" else c.kv.view(-1, 576)[:, 3]
    for j in (2, 39, 700 - T - window + 1, 700 - T - window + 2, 500, 700 - 2):
        at = c.places(b, [j])
        kept = rows[at].clone()
        rows[at] = -math.inf
        got, l2 = mla.decode_paged_window(q, qr, c.kv, c.table, n, window, sinks, SCALE, kv_scale=c.scale, return_lse=True)
        sees = window_sees(lens, T, window, sinks, 700)[b][:, j]
        assert sees.any() and all_nan(got[b][sees]) and all_nan(l2[b][sees]), j
        assert torch.equal(got[b][~sees], out[b][~sees]) and torch.equal(l2[b][~sees], lse[b][~sees]), j
        rows[at] = kept


@pytest.mark.parametrize("which", CALLS)
@pytest.mark.parametrize("flags", [0, mla.FLAG_PORTABLE_KERNEL])
@pytest.mark.parametrize("kind, d_c", [("bf16", 512), ("bf16", 256), ("fp8", 512), ("fp8", 256), ("f32", 512)])
def test_an_infinite_query_is_nan_and_nobody_else_is(kind, d_c, flags, which):
    """Also where all of its scores are -inf: the rows' values at that place have one sign."""
    call, out, lse, c, (q, qr), b, n = tree_call(kind, which, flags, d_c)
    if kind == "fp8":
        codes = c.kv.view(torch.uint8).view(-1, d_c + 64)
        codes[:, 3] = torch.where((codes[:, 3] & 127) == 127, codes[:, 3], (codes[:, 3] & 127).clamp(min=1))
    else:
        c.kv.view(-1, d_c + 64)[:, 3].abs_()
    ref, l0 = call()
    kept = q.clone()
    for t, h, what in ((0, 3, math.inf), (out.shape[1] - 1, out.shape[2] - 1, -math.inf)):
        q[b, t, h, 3] = what
        got, l2 = call()
        assert all_nan(got[b, t, h]) and all_nan(l2[b, t, h])
        got[b, t, h], l2[b, t, h] = ref[b, t, h], l0[b, t, h]
        assert torch.equal(got, ref) and torch.equal(l2, l0)
        q.copy_(kept)


# ------------------------------------------------------------------ prompts

# (length, tokens, heads, window, sinks, d_c): keys and values by the kernel that keeps a head's weights and by the one that streams them, keys whole and in chunks
PROMPTS = [(520, 300, 2, 90, 4, 256), (520, 300, 2, 90, 40, 512), (4500, 130, 2, 4200, 70, 512), (2760, 200, 64, 900, 33, 512), (2760, 200, 64, 900, 33, 256)]


def prompt(L, T, H, window, sinks, d_c):
    g, c = gen(L + d_c), Cache([L], d_c, 64, 64, BF, 3)
    qn, qr = (torch.randn((1, T, H, d), generator=g, device=DEV).to(BF) for d in (128, 64))
    UK, UV = ((torch.randn(s, generator=g, device=DEV) * d_c ** -0.5).to(BF) for s in ((H, 128, d_c), (H, d_c, 128)))
    n = torch.tensor([L], dtype=torch.int32, device=DEV)
    call = lambda: [x[0] for x in mla.prefill_window(qn, qr, UK, UV, c.kv, c.table, n, window, sinks, SCALE, return_lse=True)]
    call.q_rope = qr
    # a row of the first ones, one that only some of the tokens see for its age, one that everybody sees (if the window is wide enough), new ones
    rows = [1, sinks - 1, L - T - window + T // 2, L - T - window + T - 1, L - window - 3, L - T - 1, L - T + 10, L - T // 2, L - 1]
    return call, c, (UK, UV), [j for j in dict.fromkeys(rows) if j >= 0], lambda j: window_sees([L], T, window, sinks, L)[0][:, j]


@pytest.mark.parametrize("size", PROMPTS)
@pytest.mark.parametrize("what", [3e38, -2.0 ** 100])
def test_a_row_whose_values_do_not_fit_reaches_nobody_who_does_not_see_it(size, what):
    """Its keys are small, and so are the scores: W_UK has little to do with the one large latent.  Its values are past bf16's range."""
    call, c, (UK, UV), rows, sees = prompt(*size)
    UK[:, :, 9] = 2.0 ** -120
    UV[:, 9] = 2.0 ** 40
    c.kv[:, :, 9] = torch.where(torch.isnan(c.kv[:, :, 9]), c.kv[:, :, 9], torch.zeros_like(c.kv[:, :, 9]))
    out, lse = call()
    assert torch.isfinite(out.float()).all()
    for j in rows:
        at = c.places(0, [j])
        c.kv.view(-1, c.kv.shape[2])[at, 9] = what
        got, l2 = call()
        s = sees(j)
        assert torch.equal(got[~s], out[~s]) and torch.equal(l2[~s], lse[~s]), j
        assert s.any() and all_nan(got[s]) and all_nan(l2[s]), j
        c.kv.view(-1, c.kv.shape[2])[at, 9] = 0.0


@pytest.mark.parametrize("size", PROMPTS)
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_a_latent_that_is_not_finite_reaches_whoever_sees_it(size, what):
    """Where 32 query rows beside each other all see it and where some do, new rows and old ones."""
    call, c, _, rows, sees = prompt(*size)
    out, lse = call()
    for j in rows:
        at = c.places(0, [j])
        kept = c.kv.view(-1, c.kv.shape[2])[at].clone()
        c.kv.view(-1, c.kv.shape[2])[at, 9] = what
        s = sees(j)
        for _ in range(2):
            got, l2 = call()
            assert torch.equal(got[~s], out[~s]) and torch.equal(l2[~s], lse[~s]), j
            assert s.any() and all_nan(got[s]) and all_nan(l2[s]), j
        c.kv.view(-1, c.kv.shape[2])[at] = kept


def test_a_large_latent_below_the_limit_is_a_number():
    call, c, (UK, UV), rows, sees = prompt(520, 300, 2, 90, 4, 256)
    UK[:, :, 9] = 2.0 ** -100
    UV[:, 9] = 2.0 ** -100
    for j in rows:
        c.kv.view(-1, 320)[c.places(0, [j]), 9] = 2.0 ** 99
    out, lse = call()
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("size", PROMPTS)
def test_a_rope_part_that_is_not_finite(size):
    """Scores of +inf make NaN, also of the log-sum-exp, those of -inf count for nothing; whoever does not see the row keeps the bits."""
    call, c, _, rows, sees = prompt(*size)
    d_c = size[-1]
    out, lse = call()
    for j in rows:
        at = c.places(0, [j])
        kept = c.kv.view(-1, d_c + 64)[at].clone()
        c.kv.view(-1, d_c + 64)[at, d_c + 5] = math.inf
        up, s = call.q_rope[0, :, :, 5] > 0, sees(j)[:, None]
        got, l2 = call()
        assert torch.equal(got[~s[:, 0]], out[~s[:, 0]]) and torch.equal(l2[~s[:, 0]], lse[~s[:, 0]]), j
        assert all_nan(got[s & up]) and all_nan(l2[s & up]), j
        # (2 s_err of a weight left out, and half a step of bf16 on the normaliser: far below 0.02)
        assert torch.isfinite(got[s & ~up].float()).all() and torch.isfinite(l2[s & ~up]).all() and (l2[s & ~up] <= lse[s & ~up] + 0.02).all(), j
        c.kv.view(-1, d_c + 64)[at] = kept
