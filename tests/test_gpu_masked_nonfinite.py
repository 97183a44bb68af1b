"""Committed rows that are not finite, in tiles that every token of the call sees whole (tests/test_gpu_masked.py has them in drafted
rows and at a window's edge): the tokens that see such a row are NaN, on every kernel and whichever tile it lies in."""
import math

import pytest
import torch

from paper_2502_07864_amd import mla
from test_gpu_masked import BF, DEV, SCALE, run_tree
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
