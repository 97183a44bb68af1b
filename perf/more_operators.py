"""Masked attention over the latent cache, and the rows that a drafted tree leaves in it, as timed cases.

``tree``     tokens of a drafted tree over a paged cache, absorbed form: every token sees the committed rows and, of the
             drafted ones, those that its mask names (``mla.decode_paged_tree``).
``window``   one or a few new tokens with a sliding window and a few first rows that stay visible, absorbed form
             (``mla.decode_paged_window``).
``prefill``  prompts, or chunks of them, under the same window, keys and values per head (``mla.prefill_window``).
``move``     rows of accepted tokens moved to where the next step expects them (``layer.cache_move``).

``listed`` names twelve cases, ``draw`` gives others of the same ranges.  Every operator is written three times: the
calls of the framework, plain tensor operations in 32 bits, and its definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False        # True: run() makes the framework's calls; False: the plain form

DEV = "cuda:0"
D_ROPE = 64
D_HEAD = 128
SCALE = (D_HEAD + D_ROPE) ** -0.5
E4M3_MAX = 448.0
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "f32": 4, "fp8": 1}


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------

def _tree(batch, tokens, heads, context, d_c=512, cache="bf16", page=64, ragged=False, width=8, io="bf16"):
    return dict(kind="tree", batch=batch, tokens=tokens, heads=heads, context=context, d_c=d_c, cache=cache, page=page,
                ragged=ragged, width=width, io=io)


def _window(batch, tokens, heads, context, window, sinks, d_c=512, cache="bf16", page=64, ragged=False, io="bf16"):
    return dict(kind="window", batch=batch, tokens=tokens, heads=heads, context=context, window=window, sinks=sinks, d_c=d_c,
                cache=cache, page=page, ragged=ragged, io=io)


def _prefill(batch, tokens, heads, context, window, sinks, d_c=512, ragged=False):
    return dict(kind="prefill", batch=batch, tokens=tokens, heads=heads, context=context, window=window, sinks=sinks, d_c=d_c,
                ragged=ragged)


def _move(batch, tokens, accepted, context, d_c=512, cache="bf16", page=64):
    return dict(kind="move", batch=batch, tokens=tokens, accepted=accepted, context=context, d_c=d_c, cache=cache, page=page)


def listed():
    return [
        # one interactive user and a small tree behind a short conversation: the smallest call, where latency counts
        dict(name="tree_b1_1k", **_tree(1, 8, 32, 1000)),
        # a decode batch on the headline cache, sixteen drafted tokens each
        dict(name="tree_b16_8k", **_tree(16, 16, 32, 8192)),
        # long sequences on the fp8 cache, an odd tree
        dict(name="tree_fp8_b4_128k", **_tree(4, 31, 32, 131072, cache="fp8")),
        # many sequences of different lengths, the smaller layer, wide trees
        dict(name="tree_h28_b64_ragged", **_tree(64, 63, 28, 4096, d_c=256, ragged=True)),
        # one long stream, one token: what a window is for
        dict(name="window_b1_128k", **_window(1, 1, 32, 131072, 4096, 4)),
        # a large decode batch of different lengths, one token each
        dict(name="window_b64_ragged", **_window(64, 1, 32, 32768, 4096, 4, ragged=True)),
        # a few drafted tokens in a line, fp8 cache, a short window, an odd batch
        dict(name="window_fp8_b15_mtp4", **_window(15, 4, 28, 16384, 1024, 4, cache="fp8")),
        # a short question behind a long document
        dict(name="prefill_window_b2_136", **_prefill(2, 136, 28, 10539, 4096, 4, d_c=256)),
        # one chunk of eight prompts in flight
        dict(name="prefill_window_chunk_b8", **_prefill(8, 500, 28, 6000, 1024, 4, d_c=256, ragged=True)),
        # whole prompts
        dict(name="prefill_window_b4_8k", **_prefill(4, 8192, 32, 8192, 1024, 4)),
        # one user's accepted tokens
        dict(name="move_b1", **_move(1, 24, 3, 1000)),
        # a large batch's, on the fp8 cache
        dict(name="move_fp8_b64", **_move(64, 64, 8, 8192, cache="fp8")),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _count(rng, lo, hi):
    """Any odd number, or a power of two."""
    n = _log(rng, lo, hi)
    return n | 1 if rng.random() < 0.6 else 1 << max(lo, n).bit_length() - 1


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "window", "window", "window", "prefill", "prefill", "prefill", "move"])
    d_c, page = rng.choice([256, 512, 512]), rng.choice([64, 64, 64, 16, 32, 128])
    cache, io = rng.choice([("bf16", "bf16")] * 5 + [("fp8", "bf16")] * 3 + [("f32", "f32")])
    heads = rng.choice([8, 16, 20, 28, 32, 32, 40, 64])
    top = max(work(c)["flops"] for c in listed() if c["kind"] == kind)
    for _ in range(1000):
        if kind == "tree":
            batch, tokens, context = _count(rng, 1, 64), min(_count(rng, 1, 64), 64), _log(rng, 17, 131072)
            if cache == "f32":
                batch, context = min(batch, 4), min(context, 2048)
            c = _tree(batch, tokens, heads, context, d_c, cache, page, rng.random() < 0.5, rng.choice([2, 4, 8, 16]), io)
        elif kind == "window":
            batch, tokens, context = _count(rng, 1, 64), rng.choice([1, 1, 1, 2, 3, 4, 7]), _log(rng, 17, 131072)
            window, sinks = _log(rng, 33, 8192), rng.choice([0, 1, 4, 4, 4, 64, 100])
            if cache == "f32":
                batch, window = min(batch, 4), min(window, 2048)
            c = _window(batch, min(tokens, context), heads, context, window, sinks, d_c, cache, page, rng.random() < 0.5, io)
        elif kind == "prefill":
            batch, tokens = _log(rng, 1, 16), _count(rng, 65, 8192)
            context = rng.choice([tokens, _log(rng, tokens, 4 * tokens + 4096)])
            c = _prefill(batch, tokens, rng.choice([8, 20, 28, 32]), context, _log(rng, 64, 8192), rng.choice([0, 1, 4, 4, 64, 100]), d_c,
                         rng.random() < 0.5)
        else:
            tokens = rng.choice([24, 33, 48, 64])
            c = _move(_count(rng, 1, 64), tokens, rng.choice([2, 3, 4, 5, 6]), _log(rng, 17, 131072), d_c, cache, page)
        # (the rows that a pass reads, in the pool: at most as many as the largest listed case's)
        rows = c["batch"] * (c["context"] if kind in ("tree", "prefill") else 0)
        if work(c)["flops"] <= top and rows <= 600000:
            return c
    raise AssertionError("no case in range")


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std


def _host(case, seed):
    """Lengths, tree parents and accepted paths: small whole numbers made on the host.  The sizes that `work` counts come
    from the case alone (seed 0); a seed moves what it may without changing them."""
    return random.Random((seed, case["kind"], case["batch"], case["tokens"], case["context"]).__repr__())


def _lengths(c):
    """Committed rows (tree, move) or rows with the new ones counted (window, prefill) of every sequence."""
    rng = _host(c, 0)
    if not c.get("ragged"):
        return [c["context"]] * c["batch"]
    low = max(1, c["context"] // 8) if c["kind"] == "tree" else max(c["tokens"], c["context"] // 8)
    return [rng.randint(min(low, c["context"]), c["context"]) for _ in range(c["batch"])]


def _masks(c, seed):
    """One drafted tree per sequence: a node's parent lies among the `width` before it; row i names i and its ancestors."""
    rng = _host(c, seed)
    trees = []
    for _ in range(c["batch"]):
        rows = []
        for i in range(c["tokens"]):
            up = rng.randint(max(-1, i - c["width"]), i - 1) if i else -1
            rows.append((rows[up] if up >= 0 else 0) | 1 << i)
        trees.append(rows)
    return trees


def _signed(rows):
    return [[v - (1 << 64) if v >> 63 else v for v in r] for r in rows]


def _pages_used(c, length):
    """Logical pages of a sequence of `length` rows that a pass may read or write."""
    page, kind = c["page"] if "page" in c else 64, c["kind"]
    if kind == "tree":
        return range(0, -(-(length + c["tokens"]) // page))
    if kind == "move":
        return range(length // page, -(-(length + c["tokens"]) // page))
    first = max(0, length - c["tokens"] - c["window"] + 1) // page
    sinks = -(-min(c["sinks"], length) // page)
    return sorted(set(range(0, sinks)) | set(range(first, -(-length // page))))


def _table(c, g):
    """(page table [B, pages], number of pages in the pool): pages in random order, -1 where a page is not needed."""
    lens, page = _lengths(c), c.get("page", 64)
    extra = c["tokens"] if c["kind"] in ("tree", "move") else 0
    width = -(-(c["context"] + extra) // page)
    used = [_pages_used(c, n) for n in lens]
    total = sum(len(u) for u in used)
    ids = torch.randperm(total, generator=g, device=DEV).cpu().tolist()
    table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
    for b, u in enumerate(used):
        table[b, list(u)] = torch.tensor(ids[at:at + len(u)], dtype=torch.int32)
        at += len(u)
    return table.to(DEV), total


def _pool(c, g, pages):
    """Cache rows: latents and rotated rope parts, both of unit variance; fp8 rows with a scale per row."""
    page, row = c.get("page", 64), c["d_c"] + D_ROPE
    cache = c.get("cache", "bf16")
    kv = torch.empty((pages, page, row), dtype=_TYPES[cache], device=DEV)
    kv_scale = torch.empty((pages, page), dtype=torch.float32, device=DEV) if cache == "fp8" else None
    step = max(1, (1 << 26) // (page * row))
    for i in range(0, pages, step):
        x = _normal(g, (min(step, pages - i), page, row))
        if cache == "fp8":
            scale = x.abs().amax(-1) / E4M3_MAX
            kv_scale[i:i + step] = scale
            x = (x / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX)
        kv[i:i + step] = x.to(kv.dtype)
    return kv, kv_scale


def prepare(case, seed):
    c, g = case, _gen(seed)
    kind, B, T = c["kind"], c["batch"], c["tokens"]
    lens = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    table, pages = _table(c, g)
    kv, kv_scale = _pool(c, g, pages)
    s = dict(case=c, kv=kv, kv_scale=kv_scale, table=table, lens=lens)
    if kind == "move":
        # trees drafted level by level, eight wide, the likeliest node first: the first token of the accepted path is at its
        # place already, the others lie behind all the places that are written
        rng, n = _host(c, seed), c["accepted"]
        wide = 8 if T >= 8 * n else T // n
        path = [[0] + [d * wide + rng.randrange(max(0, n - d * wide), wide) for d in range(1, n)] for _ in range(B)]
        base = lens.cpu()[:, None]
        s["src"] = (base + torch.tensor(path, dtype=torch.int32)).to(DEV)
        s["dst"] = (base + torch.arange(n, dtype=torch.int32)).to(DEV)
        return s
    H, d_c, io = c["heads"], c["d_c"], _TYPES[c.get("io", "bf16")]
    s["q_rope"] = _normal(g, (B, T, H, D_ROPE)).to(io)
    if kind == "prefill":
        s["q_nope"] = _normal(g, (B, T, H, D_HEAD)).to(io)
        s["W_UK"] = _normal(g, (H, D_HEAD, d_c), d_c ** -0.5).to(io)
        s["W_UV"] = _normal(g, (H, d_c, D_HEAD), d_c ** -0.5).to(io)
        s["out"] = torch.empty((B, T, H, D_HEAD), dtype=io, device=DEV)       # (what a layer takes from a prompt)
    else:
        # (unit variance of the scaled scores, as absorbed queries of unit variance have it)
        s["q_abs"] = _normal(g, (B, T, H, d_c), (D_HEAD / d_c) ** 0.5).to(io)
        s["out"] = torch.empty((B, T, H, d_c), dtype=io, device=DEV)
        s["lse"] = torch.empty((B, T, H), dtype=torch.float32, device=DEV)
    if kind == "tree":
        s["mask"] = torch.tensor(_signed(_masks(c, seed)), dtype=torch.int64, device=DEV)
    s["ws"] = None
    if own:            # the scratch that a serving loop keeps
        from paper_2502_07864_amd import mla
        if kind == "tree":
            n = mla.decode_tree_workspace_bytes(B, T, H, d_c, table.shape[1] * c["page"])
        elif kind == "window":
            n = mla.decode_window_workspace_bytes(B, T, H, d_c, table.shape[1] * c["page"], c["window"], c["sinks"])
        else:
            n = mla.prefill_window_workspace_bytes(B, T, H, d_c, table.shape[1], c["window"], c["sinks"])
        s["ws"] = torch.empty(max(256, n), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2502_07864_amd import layer, mla
    c = s["case"]
    kind = c["kind"]
    if kind == "tree":
        mla.decode_paged_tree(s["q_abs"], s["q_rope"], s["kv"], s["table"], s["lens"], s["mask"], SCALE, kv_scale=s["kv_scale"],
                              workspace=s["ws"], out=s["out"], lse=s["lse"])
    elif kind == "window":
        mla.decode_paged_window(s["q_abs"], s["q_rope"], s["kv"], s["table"], s["lens"], c["window"], c["sinks"], SCALE,
                                kv_scale=s["kv_scale"], workspace=s["ws"], out=s["out"], lse=s["lse"])
    elif kind == "prefill":
        mla.prefill_window(s["q_nope"], s["q_rope"], s["W_UK"], s["W_UV"], s["kv"], s["table"], s["lens"], c["window"], c["sinks"],
                           SCALE, workspace=s["ws"], out=s["out"])
        return {"out": s["out"]}
    else:
        layer.cache_move(s["kv"], s["table"], s["src"], s["dst"], kv_scale=s["kv_scale"])
        return {"kv": s["kv"], "kv_scale": s["kv_scale"]}
    return {"out": s["out"], "lse": s["lse"]}


def _flat(s, at):
    """Row of the flat pool of logical positions at [B, n] (0 where a position has no page)."""
    page = s["kv"].shape[1]
    ids = s["table"].long().gather(1, (at // page).clamp(0, s["table"].shape[1] - 1))
    return (ids * page + at % page).clamp_min(0)


def _columns(c, lens):
    """Logical positions [B, n] that some token of a sequence may see: all of them, or the sinks and the window's."""
    B, T, device = c["batch"], c["tokens"], lens.device
    if c["kind"] == "tree":
        return torch.arange(c["context"] + T, device=device).expand(B, -1)
    reach = min(c["context"], c["window"] + T - 1)
    tail = lens.long()[:, None] - reach + torch.arange(reach, device=device)
    head = torch.arange(min(c["sinks"], c["context"]), device=device).expand(B, -1)
    # (a sink that the tail holds too is left to the tail)
    head = torch.where(head < lens.long()[:, None] - reach, head, torch.full_like(head, -1))
    return torch.cat((head, tail), 1)


def _sees(s, at):
    """Whether token i of sequence b sees the row at logical position at[b, j]: [B, T, n]."""
    c, lens = s["case"], s["lens"].long()
    T = c["tokens"]
    i = torch.arange(T, device=at.device)
    if c["kind"] == "tree":
        node = at - lens[:, None]
        bit = (s["mask"][:, :, None] >> node.clamp(0, 63)[:, None, :]) & 1
        return (node < 0)[:, None, :] | ((node >= 0) & (node < T))[:, None, :] & (bit != 0)
    own_at = (lens[:, None] - T + i)[:, :, None]
    j = at[:, None, :]
    return (j >= 0) & (j <= own_at) & ((j > own_at - c["window"]) | (j < c["sinks"]))


def _rows(s, at, dtype):
    """Cache rows [B, n, row] in `dtype`, rows without a place zero."""
    row = s["kv"].shape[-1]
    f = _flat(s, at)
    if s["kv_scale"] is not None:
        x = s["kv"].view(torch.uint8).view(-1, row)[f].view(torch.float8_e4m3fn).to(dtype)
        return x * s["kv_scale"].view(-1)[f].to(dtype)[..., None]
    return s["kv"].view(-1, row)[f].to(dtype)


def _softmax(x):
    """(weights not yet divided, their sums, log of the sum of exponentials) over the last axis."""
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (x - top).exp()
    z = p.sum(-1, keepdim=True)
    return p, z, (top + z.log()).squeeze(-1)


def _run_plain(s):
    c = s["case"]
    kind, B, T = c["kind"], c["batch"], c["tokens"]
    if kind == "move":
        row = s["kv"].shape[-1]
        kv = s["kv"].view(torch.uint8) if c["cache"] == "fp8" else s["kv"]
        src, dst = _flat(s, s["src"].long()).view(-1), _flat(s, s["dst"].long()).view(-1)
        kv.view(-1, row)[dst] = kv.view(-1, row)[src]
        if s["kv_scale"] is not None:
            s["kv_scale"].view(-1)[dst] = s["kv_scale"].view(-1)[src]
        return {"kv": s["kv"], "kv_scale": s["kv_scale"]}
    H, d_c = c["heads"], c["d_c"]
    at = _columns(c, s["lens"])
    sees = _sees(s, at)
    if kind == "prefill":
        out = torch.empty_like(s["out"])
        for b in range(B):
            one = dict(s, table=s["table"][b:b + 1])
            x = _rows(one, at[b:b + 1], torch.float32)[0]
            for h in range(H):
                k = torch.cat((torch.mm(x[:, :d_c], s["W_UK"][h].float().t()), x[:, d_c:]), 1)
                v = torch.mm(x[:, :d_c], s["W_UV"][h].float())
                q = torch.cat((s["q_nope"][b, :, h].float(), s["q_rope"][b, :, h].float()), 1)
                p, z, _ = _softmax((torch.mm(q, k.t()) * SCALE).masked_fill_(~sees[b], -math.inf))
                out[b, :, h] = (torch.mm(p, v) / torch.where(z > 0, z, torch.ones_like(z))).to(out.dtype)
        return {"out": out}
    x = _rows(s, at, torch.float32)
    q = torch.cat((s["q_abs"].float(), s["q_rope"].float()), -1).view(B, T * H, -1)
    scores = torch.bmm(q, x.transpose(1, 2).contiguous()).view(B, T, H, -1) * SCALE
    p, z, lse = _softmax(scores.masked_fill_(~sees[:, :, None], -math.inf))
    out = torch.bmm(p.view(B, T * H, -1), x[..., :d_c].contiguous()).view(B, T, H, d_c) / torch.where(z > 0, z, torch.ones_like(z))
    return {"out": out.to(s["out"].dtype), "lse": lse}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------

def _exact_visible(c, seed, b, length):
    """(rows in the order of their positions, [tokens, rows] of truth values) for one sequence, from the definition."""
    T = c["tokens"]
    if c["kind"] == "tree":
        allowed = torch.zeros((T, length + T), dtype=torch.bool)
        allowed[:, :length] = True
        for i, m in enumerate(_masks(c, seed)[b]):
            for k in range(T):
                allowed[i, length + k] = bool(m >> k & 1)
        return torch.arange(length + T), allowed
    first = max(0, length - T - c["window"] + 1)
    rows = torch.cat((torch.arange(min(c["sinks"], first)), torch.arange(first, length)))
    token = torch.arange(length - T, length)[:, None]
    age = token - rows
    return rows, (age >= 0) & ((age < c["window"]) | (rows < c["sinks"]))


def exact(case, seed):
    s, c = prepare(case, seed), case
    kind, page, lens = c["kind"], c.get("page", 64), _lengths(c)
    if kind == "move":
        kv, kv_scale = s["kv"].double(), None if s["kv_scale"] is None else s["kv_scale"].double()
        before, scale_before = kv.clone(), None if kv_scale is None else kv_scale.clone()
        place = lambda b, j: (int(table[b, j // page]), j % page)
        table, src, dst = s["table"].cpu(), s["src"].cpu().tolist(), s["dst"].cpu().tolist()
        for b in range(c["batch"]):
            for i, j in zip(src[b], dst[b]):
                kv[place(b, j)] = before[place(b, i)]
                if kv_scale is not None:
                    kv_scale[place(b, j)] = scale_before[place(b, i)]
        return {"kv": kv, "kv_scale": kv_scale}
    T, H, d_c = c["tokens"], c["heads"], c["d_c"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty((c["batch"], T, H), dtype=torch.float64, device=DEV)
    for b, length in enumerate(lens):
        rows, allowed = _exact_visible(c, seed, b, length)
        rows, allowed = rows.to(DEV), allowed.to(DEV)
        ids = s["table"][b].long()[rows // page]
        x = s["kv"][ids, rows % page].double()
        if s["kv_scale"] is not None:
            x = x * s["kv_scale"][ids, rows % page].double()[:, None]
        latent, rope = x[:, :d_c].contiguous(), x[:, d_c:].contiguous()
        blocked = torch.zeros(allowed.shape, dtype=torch.float64, device=DEV).masked_fill_(~allowed, -math.inf)
        for h in range(H):
            turned = s["q_rope"][b, :, h].double()
            if kind == "prefill":
                keys, values = latent @ s["W_UK"][h].double().t(), latent @ s["W_UV"][h].double()
                scores = s["q_nope"][b, :, h].double() @ keys.t() + turned @ rope.t()
            else:
                values = latent
                scores = s["q_abs"][b, :, h].double() @ latent.t() + turned @ rope.t()
            scores = scores * SCALE + blocked
            lse[b, :, h] = torch.logsumexp(scores, 1)
            out[b, :, h] = torch.exp(scores - lse[b, :, h, None]) @ values
    return {"out": out} if kind == "prefill" else {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    kind, T, page = c["kind"], c["tokens"], c.get("page", 64)
    row = c["d_c"] + D_ROPE
    row_bytes = row * _BYTES[c.get("cache", "bf16")] + 4 * (c.get("cache") == "fp8")
    if kind == "move":
        n = c["batch"] * (c["accepted"] - 1)
        return {"bytes": n * 2 * row_bytes + c["batch"] * c["accepted"] * 8, "flops": n}
    H, d_c, io = c["heads"], c["d_c"], _BYTES[c.get("io", "bf16")]
    rows = pairs = 0                     # cached rows that are read, and (token, row) pairs that are scored
    for b, length in enumerate(_lengths(c)):
        if kind == "tree":
            rows += length + T
            pairs += T * length
        else:
            first = max(0, length - T - c["window"] + 1)
            rows += min(c["sinks"], first) + length - first
            for at in range(length - T, length):
                start = max(0, at - c["window"] + 1)
                pairs += min(c["sinks"], start) + at + 1 - start
    if kind == "tree":                   # (of the drafted rows, each token's own and its ancestors')
        pairs += sum(bin(m).count("1") for t in _masks(c, 0) for m in t)
    tokens = c["batch"] * T * H
    if kind == "prefill":
        return {"bytes": rows * row_bytes + tokens * (2 * D_HEAD + D_ROPE) * io + 2 * H * D_HEAD * d_c * io,
                "flops": 4 * d_c * D_HEAD * rows * H + 2 * (2 * D_HEAD + D_ROPE) * pairs * H}
    return {"bytes": rows * row_bytes + tokens * ((row + d_c) * io + 4) + (8 * c["batch"] * T if kind == "tree" else 0),
            "flops": 2 * (row + d_c) * pairs * H}
