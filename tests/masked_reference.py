"""Masked attention over a paged latent cache in 64 bits, from a table of truth values, and bounds for what a kernel may be off.

The bounds count roundings (u = 2^-24 for fp32, h = 2^-8 for bf16, half a step of either), for each output by itself:

* a score is a dot product of n terms in fp32, scaled: off by at most s_err = (n + 8) u scale sum|q||k|, plus 4 u |s| for the
  change to powers of two; a weight is then off by the factor 1 +- 2 s_err (s_err stays below 0.01), and 8 u for the exponential;
* bf16 io rounds every weight of the value sum once (h), every partial result once where chunks are merged (h) and the
  result (h); sums of N positive fp32 terms are off by at most N u;
* so |o - o64| <= A (2 s_err + 8 u + 2 N u + 2 h) + h |o64| with A = sum_j p_j |v_j| (without the h for fp32 io), and
  |lse - lse64| <= s_err + 8 u + N u + 4 u (1 + max|s|);
* prompts: keys and values are rounded to bf16 per head: k off by h |k| and (d_c + 8) u sum|W||c|, so s_err gains
  scale sum|q| |dk|, and A the values' own h.
"""
import torch

U, H = 2.0 ** -24, 2.0 ** -8


def gather(kv, kv_scale, page_table, n):
    """Rows 0 .. n - 1 of every sequence in fp64 [B, n, row], rows without a page zero, and which have one [B, n]."""
    page, row = kv.shape[1], kv.shape[2]
    at = torch.arange(n, device=kv.device)
    col = (at // page).clamp(max=page_table.shape[1] - 1)
    ids = page_table.long()[:, col]
    there = (ids >= 0) & (ids < kv.shape[0]) & (at < page * page_table.shape[1])
    flat = torch.where(there, ids, torch.zeros_like(ids)) * page + at % page
    x = kv.double().view(-1, row)[flat]
    if kv_scale is not None:
        x = x * kv_scale.double().view(-1)[flat][..., None]
    return x, there


def attend(q, k, v, sees, scale, bf16, dk=None, dv=None, terms=None):
    """q [T, H, d], k [n, d] or [H, n, d], v likewise, sees [T, n]; (o, lse, bound of o, bound of lse).  Rows nobody sees are
    not multiplied."""
    T, Hh, d = q.shape
    o = torch.zeros((T, Hh, v.shape[-1]), dtype=torch.float64, device=q.device)
    lse = torch.full((T, Hh), -torch.inf, dtype=torch.float64, device=q.device)
    eo, el = torch.zeros_like(o), torch.zeros_like(lse)
    for t in range(T):
        rows = sees[t].nonzero()[:, 0]
        if rows.numel() == 0:
            continue
        kk, vv = (x[rows] if x.dim() == 2 else x[:, rows] for x in (k, v))
        kk, vv = (x.expand(Hh, *x.shape) if x.dim() == 2 else x for x in (kk, vv))
        s = torch.bmm(kk, q[t][:, :, None])[..., 0] * scale
        size = torch.bmm(kk.abs(), q[t].abs()[:, :, None])[..., 0] * abs(scale)
        err = ((terms or d) + 8) * U * size + 4 * U * s.abs()
        if dk is not None:
            err = err + abs(scale) * torch.bmm(dk[:, rows], q[t].abs()[:, :, None])[..., 0]
        err = err.amax(1)
        lse[t] = torch.logsumexp(s, 1)
        p = (s - lse[t][:, None]).exp()[:, None]
        o[t] = torch.bmm(p, vv)[:, 0]
        A = torch.bmm(p, vv.abs())[:, 0]
        N = rows.numel()
        eo[t] = A * (2 * err + 8 * U + 2 * N * U + (2 * H if bf16 else 0.0))[:, None] + (H if bf16 else U) * o[t].abs() + 1e-30
        if dv is not None:
            eo[t] += torch.bmm(p, dv[:, rows])[:, 0]
        el[t] = err + 8 * U + N * U + 4 * U * (1 + s.abs().amax(1))
    return o, lse, eo, el


def close(got, want, bound, what):
    got = got.double()
    assert torch.equal(torch.isneginf(got), torch.isneginf(want)), f"{what}: -inf in other places"
    live = ~torch.isneginf(want)
    off = (got - want).abs()[live] - bound[live]
    assert not torch.isnan(off).any(), f"{what}: NaN"
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {off.max().item():.3e} beyond the bound"
