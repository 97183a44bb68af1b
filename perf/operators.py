"""The operators around the latent attention of one layer, as timed cases.

``norm``   RMS norm of the hidden states, usually with the residual's addition, to the layer's type and / or to
           e4m3 codes with one scale per token and 128 columns (``layer.rms_norm``, ``layer.rms_norm_fp8``).
``quant``  the same codes and scales of a tensor as it is: what the attention returns, before the output
           projection (``layer.quantize_rows``).
``gemm``   a projection on such codes: e4m3 x e4m3, one scale per token and 128 input columns on the left, one per
           128 x 128 block on the right (``layer.gemm_fp8``).
``rope``   the queries' rows [nope | rope] taken apart and their rope part rotated (``layer.rope_queries``).
``store``  rows [c | k] of new tokens, k rotated, c with an RMS norm of its own or as it is, rounded to the cache's
           type and written through the page table (``layer.cache_store``).

``listed`` names twelve cases, ``draw`` gives others of the same ranges.  Every operator is written three times: the
calls of the framework, plain tensor operations in 32 bits, and its definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False        # True: run() makes the framework's calls; False: the plain form

DEV = "cuda:0"
BLOCK = 128        # columns per scale
D_ROPE = 64
E4M3_MAX = 448.0
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "f32": 4, "fp8": 1}


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------

def _norm(tokens, dim, io="bf16", residual=True, codes=True, plain=False):
    return dict(kind="norm", tokens=tokens, dim=dim, io=io, residual=residual, codes=codes, plain=plain)


def _quant(tokens, dim, io="bf16"):
    return dict(kind="quant", tokens=tokens, dim=dim, io=io)


def _gemm(tokens, n, k, out="bf16"):
    return dict(kind="gemm", tokens=tokens, n=n, k=k, out=out)


def _rope(tokens, heads, d_nope=128, d_rope=D_ROPE, io="bf16", half=False, scaling="none", context=8192):
    return dict(kind="rope", tokens=tokens, heads=heads, d_nope=d_nope, d_rope=d_rope, io=io, half=half, scaling=scaling, context=context)


def _store(batch, new, context, d_c=512, io="bf16", cache="bf16", half=False, scaling="none", norm=False, page=64):
    return dict(kind="store", batch=batch, new=new, context=context, d_c=d_c, io=io, cache=cache, half=half, scaling=scaling, norm=norm, page=page)


def listed():
    return [
        # one interactive user, model dimension 4096: the smallest call, where latency counts; the bf16 states are wanted
        # beside the codes (a bf16 cache projection reads them)
        dict(name="norm_b1", **_norm(1, 4096, plain=True)),
        # a decode batch of an odd number of sequences, the smaller layer (28 heads)
        dict(name="norm_b61_3584", **_norm(61, 3584)),
        # four whole prompts of 8192 tokens
        dict(name="norm_prompt_32k", **_norm(32768, 4096)),
        # the query projection of one token: 25 MB of weights for one row
        dict(name="gemm_q_b1", **_gemm(1, 32 * 192, 4096)),
        # the cache rows of a decode batch, 576 wide, in fp32 for the rounding to come: few columns
        dict(name="gemm_kv_b16", **_gemm(16, 576, 4096, out="f32")),
        # the output projection of an odd decode batch, the smaller layer
        dict(name="gemm_o_b61", **_gemm(61, 3584, 28 * 128)),
        # the query projection of one chunk of eight prompts, 500 tokens each: ragged tiles
        dict(name="gemm_q_chunk", **_gemm(4000, 28 * 192, 3584)),
        # the query projection of four whole prompts: the largest product
        dict(name="gemm_q_prompt", **_gemm(32768, 32 * 192, 4096)),
        # the queries of a decode batch
        dict(name="rope_b16", **_rope(16, 32)),
        # the queries of four whole prompts, the half layout with frequencies scaled for a long context
        dict(name="rope_prompt_32k", **_rope(32768, 32, half=True, scaling="yarn", context=131072)),
        # one new row for each of four long sequences on the fp8 cache, out of an fp32 projection
        dict(name="store_fp8_b4_128k", **_store(4, 1, 131072, io="f32", cache="fp8", scaling="yarn")),
        # whole prompts written to the bf16 cache, latents normed on the way
        dict(name="store_prompt_b4_8k", **_store(4, 8192, 8192, norm=True)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _count(rng, lo, hi):
    """A number of tokens: any odd one, or a power of two."""
    n = _log(rng, lo, hi)
    return n | 1 if rng.random() < 0.6 else 1 << max(lo, n).bit_length() - 1


def draw(rng):
    kind = rng.choice(["norm", "norm", "quant", "gemm", "gemm", "gemm", "gemm", "rope", "rope", "store", "store"])
    dims = [1024, 2048, 3584, 4096, 5120]
    if kind in ("norm", "quant"):
        tokens, dim = _count(rng, 1, 32000), rng.choice(dims + [_log(rng, 65, 4096) | 1])
        io = rng.choice(["bf16", "bf16", "bf16", "f32"])
        tokens = min(tokens, 32768 * 4096 // (dim * _BYTES[io]) | 1)
        if kind == "quant":
            return _quant(tokens, dim, io)
        codes = rng.random() < 0.8
        return _norm(tokens, dim, io, rng.random() < 0.8, codes, not codes or rng.random() < 0.4)
    if kind == "gemm":
        heads = rng.choice([8, 20, 28, 32, 40])
        n = rng.choice([576, 320, heads * 192, heads * 128, _log(rng, 33, 6000) | 1])
        k = rng.choice(dims + [heads * 128, 16 * rng.choice([7, 9, 33, 65, 101, 223])])
        tokens = min(_count(rng, 1, 32000), 32768 * 6144 * 4096 // (n * k))
        return _gemm(tokens, n, k, rng.choice(["bf16", "bf16", "f32"]))
    half, scaling = rng.random() < 0.5, rng.choice(["none", "linear", "yarn"])
    context = _log(rng, 500, 131072) | 1
    if kind == "rope":
        heads = rng.choice([8, 20, 28, 32, 32, 64])
        d_nope, d_rope = rng.choice([(128, 64), (128, 64), (64, 32), (0, 128), (96, 40)])
        io = rng.choice(["bf16", "bf16", "f32"])
        tokens = _count(rng, 1, 32000)
        tokens = min(tokens, 32768 * 32 * 192 * 2 // (heads * (d_nope + d_rope) * _BYTES[io]) | 1)
        return _rope(tokens, heads, d_nope, d_rope, io, half, scaling, context)
    batch = _count(rng, 1, 64)
    new = rng.choice([1, 1, 2, 3, _count(rng, 4, 8192)])
    new = max(1, min(new, context, 65536 // batch))
    cache = rng.choice(["bf16", "bf16", "fp8", "f32"])
    io = "f32" if cache == "f32" else rng.choice(["bf16", "f32"])
    return _store(batch, new, context, rng.choice([256, 512, 512, 440]), io, cache, half, scaling, rng.random() < 0.5, rng.choice([64, 64, 16, 33]))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype=torch.float32, std=1.0):
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    return (x * std if std != 1.0 else x).to(dtype)


def _hidden(g, tokens, dim, dtype):
    """Hidden states as a transformer has them: Gaussian, a few channels an order of magnitude larger."""
    x = torch.randn((tokens, dim), generator=g, device=DEV, dtype=torch.float32)
    loud = torch.randperm(dim, generator=g, device=DEV)[:4]
    x[:, loud] *= 12.0
    return x.to(dtype)


def _frequencies(d_rope, scaling, base=10000.0, factor=16.0, original=4096, beta_fast=32.0, beta_slow=1.0):
    """(radians per position of every pair in fp64, gain of the rotated part)."""
    i = torch.arange(0, d_rope, 2, dtype=torch.float64, device=DEV)
    f = base ** (-i / d_rope)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        # pairs that turn often within the trained length stay, pairs that turn less than once in it are interpolated
        at = lambda turns: d_rope * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(at(beta_fast)), 0), min(math.ceil(at(beta_slow)), d_rope // 2 - 1)
        ramp = ((i / 2 - low) / max(high - low, 1e-3)).clamp(0, 1)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _blocks(n):
    return -(-n // BLOCK)


def _by_block(x):
    """[rows, dim] -> [rows, blocks, 128], padded with zeros."""
    rows, dim = x.shape
    return torch.nn.functional.pad(x, (0, _blocks(dim) * BLOCK - dim)).view(rows, -1, BLOCK)


def _codes(x):
    """Codes of x [rows, dim] (fp32) and their scales [blocks, rows]."""
    b = _by_block(x)
    top = b.abs().amax(-1)
    scale = torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top))
    q = (b / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).view(x.shape[0], -1)[:, :x.shape[1]]
    return q.to(torch.float8_e4m3fn).contiguous(), scale.t().contiguous()


def _weight_codes(w):
    """Codes of w [n, k] (fp32) and their scales, one per 128 x 128 block."""
    n, k = w.shape
    p = torch.nn.functional.pad(w, (0, _blocks(k) * BLOCK - k, 0, _blocks(n) * BLOCK - n))
    b = p.view(_blocks(n), BLOCK, _blocks(k), BLOCK)
    scale = b.abs().amax((1, 3)) / E4M3_MAX
    q = (b / scale[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(p.shape)[:n, :k]
    return q.to(torch.float8_e4m3fn).contiguous(), scale.contiguous()


def prepare(case, seed):
    c, g = case, _gen(seed)
    kind = c["kind"]
    if kind in ("norm", "quant"):
        io = _TYPES[c["io"]]
        t, d = c["tokens"], c["dim"]
        s = dict(case=c, x=_hidden(g, t, d, io), eps=1e-5)
        if kind == "norm":
            s["weight"] = (1.0 + 0.2 * _normal(g, (d,))).to(io)
            s["residual"] = _hidden(g, t, d, io) if c["residual"] else None
            s["residual_out"] = torch.empty((t, d), dtype=io, device=DEV) if c["residual"] else None
            s["y"] = torch.empty((t, d), dtype=io, device=DEV) if c["plain"] else None
        if kind == "quant" or c["codes"]:
            s["codes"] = torch.empty((t, d), dtype=torch.float8_e4m3fn, device=DEV)
            s["scales"] = torch.empty((_blocks(d), t), dtype=torch.float32, device=DEV)
        return s
    if kind == "gemm":
        m, n, k = c["tokens"], c["n"], c["k"]
        a, a_scales = _codes(_hidden(g, m, k, torch.float32))
        w, w_scales = _weight_codes(_normal(g, (n, k), std=k ** -0.5))
        s = dict(case=c, a=a, a_scales=a_scales, w=w, w_scales=w_scales, out=torch.empty((m, n), dtype=_TYPES[c["out"]], device=DEV), ws=None)
        if own:          # the scratch that a serving loop keeps
            from paper_2502_07864_amd import layer
            s["ws"] = torch.empty(max(256, layer.gemm_fp8_workspace_bytes(m, n, k)), dtype=torch.uint8, device=DEV)
        return s
    freq, gain = _frequencies(c["d_rope"] if kind == "rope" else D_ROPE, c["scaling"])
    io = _TYPES[c["io"]]
    if kind == "rope":
        t, h = c["tokens"], c["heads"]
        return dict(
            case=c, freq=freq, gain=gain, q=_normal(g, (t, h, c["d_nope"] + c["d_rope"]), io),
            positions=torch.randint(0, c["context"], (t,), generator=g, device=DEV).to(torch.int32),
            q_nope=torch.empty((t, h, c["d_nope"]), dtype=io, device=DEV), q_rope=torch.empty((t, h, c["d_rope"]), dtype=io, device=DEV))
    # the last `new` tokens of contexts of different lengths; only their pages are in the pool
    b, new, page, row = c["batch"], c["new"], c["page"], c["d_c"] + D_ROPE
    first = torch.randint(0, c["context"] - new + 1, (b,), generator=g, device=DEV)
    positions = first[:, None] + torch.arange(new, device=DEV)
    width = -(-c["context"] // page)
    each = min(width, (new + page - 2) // page + 1)              # pages that `new` rows in a line may touch
    order = torch.randperm(b * each, generator=g, device=DEV).view(b, each).to(torch.int32)
    at = torch.arange(width, device=DEV)[None, :] - torch.minimum(first // page, torch.tensor(width - each, device=DEV))[:, None]
    table = torch.where((at >= 0) & (at < each), order.gather(1, at.clamp(0, each - 1)), torch.full_like(order[:1, :1], -1)).contiguous()
    return dict(
        case=c, freq=freq, gain=gain, rows=_normal(g, (b, new, row), io), positions=positions.to(torch.int32).contiguous(), table=table,
        weight=(1.0 + 0.2 * _normal(g, (c["d_c"],))).to(io) if c["norm"] else None, eps=1e-6,
        kv=torch.zeros((b * each, page, row), dtype=_TYPES[c["cache"]], device=DEV),
        kv_scale=torch.zeros((b * each, page), dtype=torch.float32, device=DEV) if c["cache"] == "fp8" else None)


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2502_07864_amd import layer
    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        if c["codes"]:
            layer.rms_norm_fp8(s["x"], s["weight"], s["eps"], residual=s["residual"], codes=s["codes"], scales=s["scales"],
                               residual_out=s["residual_out"], out=s["y"])
            return {"codes": s["codes"], "scales": s["scales"], "residual": s["residual_out"], "y": s["y"]}
        layer.rms_norm(s["x"], s["weight"], s["eps"], residual=s["residual"], residual_out=s["residual_out"], out=s["y"])
        return {"codes": None, "scales": None, "residual": s["residual_out"], "y": s["y"]}
    if kind == "quant":
        layer.quantize_rows(s["x"], codes=s["codes"], scales=s["scales"])
        return {"codes": s["codes"], "scales": s["scales"]}
    if kind == "gemm":
        # a bf16 output is rounded a hundred times more coarsely than the matrix cores add 8-bit products
        layer.gemm_fp8(s["a"], s["a_scales"], s["w"], s["w_scales"], out=s["out"], workspace=s["ws"],
                       flags=layer.GEMM_FAST_SUMS if c["out"] == "bf16" else 0)
        return {"out": s["out"]}
    layout = layer.ROPE_HALF if c["half"] else layer.ROPE_INTERLEAVED
    if kind == "rope":
        layer.rope_queries(s["q"], s["positions"], s["freq"], gain=s["gain"], layout=layout, q_nope=s["q_nope"], q_rope=s["q_rope"])
        return {"q_nope": s["q_nope"], "q_rope": s["q_rope"]}
    layer.cache_store(s["rows"], s["positions"], s["freq"], s["kv"], s["table"], c["d_c"], gain=s["gain"], layout=layout,
                      norm_weight=s["weight"], eps=s["eps"], kv_scale=s["kv_scale"])
    return {"kv": s["kv"], "kv_scale": s["kv_scale"]}


def _rotate(x, angles, gain, half):
    """x [..., d] turned by angles [..., d / 2] (fp64: positions reach 10^5 radians), arithmetic in x's type."""
    cs, sn = (angles.cos() * gain).to(x.dtype), (angles.sin() * gain).to(x.dtype)
    d = x.shape[-1]
    re, im = (x[..., :d // 2], x[..., d // 2:]) if half else (x[..., 0::2], x[..., 1::2])
    parts = (re * cs - im * sn, re * sn + im * cs)
    return torch.cat(parts, -1) if half else torch.stack(parts, -1).flatten(-2)


def _slots(s):
    """Row of the flat pool that every new token's row goes to."""
    page = s["case"]["page"]
    at = s["positions"].long()
    return (s["table"].long().gather(1, at // page) * page + at % page).view(-1)


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind in ("norm", "quant"):
        v = s["x"].float()
        if kind == "quant":
            codes, scales = _codes(v)
            return {"codes": codes, "scales": scales}
        if c["residual"]:
            v = v + s["residual"].float()
        y = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + s["eps"]) * s["weight"].float()
        codes, scales = _codes(y) if c["codes"] else (None, None)
        return {"codes": codes, "scales": scales, "residual": v.to(s["x"].dtype) if c["residual"] else None,
                "y": y.to(s["x"].dtype) if c["plain"] else None}
    if kind == "gemm":
        m, n, k = c["tokens"], c["n"], c["k"]
        a = s["a"].float() * s["a_scales"].t().repeat_interleave(BLOCK, 1)[:, :k]
        w = s["w"].float() * s["w_scales"].repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
        return {"out": torch.mm(a, w.t()).to(s["out"].dtype)}
    angles = s["positions"].double()[..., None] * s["freq"]
    if kind == "rope":
        q, dn = s["q"], c["d_nope"]
        return {"q_nope": q[..., :dn].contiguous(), "q_rope": _rotate(q[..., dn:].float(), angles[:, None], s["gain"], c["half"]).to(q.dtype)}
    x, dc = s["rows"].float(), c["d_c"]
    latent = x[..., :dc]
    if c["norm"]:
        latent = latent * torch.rsqrt((latent * latent).mean(-1, keepdim=True) + s["eps"]) * s["weight"].float()
    row = torch.cat((latent, _rotate(x[..., dc:], angles, s["gain"], c["half"])), -1).view(c["batch"] * c["new"], -1)
    kv, at = s["kv"], _slots(s)
    if c["cache"] == "fp8":
        top = row.abs().amax(-1)
        scale = torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top))
        codes = (row / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(kv.dtype)
        kv.view(torch.uint8).view(-1, row.shape[1])[at] = codes.view(torch.uint8)
        s["kv_scale"].view(-1)[at] = scale
    else:
        kv.view(-1, row.shape[1])[at] = row.to(kv.dtype)
    return {"kv": kv, "kv_scale": s["kv_scale"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------

def _exact_codes(y):
    """What the codes and their scales stand for before the codes' rounding."""
    rows, dim = y.shape
    scales = torch.empty((_blocks(dim), rows), dtype=torch.float64, device=y.device)
    codes = torch.empty_like(y)
    for i in range(_blocks(dim)):
        part = y[:, i * BLOCK:(i + 1) * BLOCK]
        top = part.abs().max(1).values
        top[top == 0] = E4M3_MAX
        scales[i] = top / E4M3_MAX
        codes[:, i * BLOCK:(i + 1) * BLOCK] = part / scales[i][:, None]
    return codes, scales


def _exact_turn(x, angles, gain, half):
    """The pairs of the last axis as complex numbers, turned."""
    d = x.shape[-1]
    z = torch.complex(x[..., :d // 2], x[..., d // 2:]) if half else torch.view_as_complex(x.unflatten(-1, (d // 2, 2)).contiguous())
    z = z * torch.polar(torch.full_like(angles, gain), angles)
    return torch.cat((z.real, z.imag), -1) if half else torch.view_as_real(z).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    kind = c["kind"]
    if kind in ("norm", "quant"):
        v = s["x"].double()
        if kind == "quant":
            codes, scales = _exact_codes(v)
            return {"codes": codes, "scales": scales}
        if c["residual"]:
            v += s["residual"].double()
        y = v / (v.square().sum(1, keepdim=True) / c["dim"] + s["eps"]).sqrt() * s["weight"].double()
        codes, scales = _exact_codes(y) if c["codes"] else (None, None)
        return {"codes": codes, "scales": scales, "residual": v if c["residual"] else None, "y": y if c["plain"] else None}
    if kind == "gemm":
        m, n, k = c["tokens"], c["n"], c["k"]
        out = torch.zeros((m, n), dtype=torch.float64, device=DEV)
        rows = torch.arange(n, device=DEV) // BLOCK
        for i in range(_blocks(k)):
            at = slice(i * BLOCK, min(k, (i + 1) * BLOCK))
            a = s["a"][:, at].double() * s["a_scales"][i].double()[:, None]
            w = s["w"][:, at].double() * s["w_scales"][rows, i].double()[:, None]
            out.addmm_(a, w.t())
        return {"out": out}
    if kind == "rope":
        q, dn = s["q"].double(), c["d_nope"]
        angles = (s["positions"].double()[:, None] * s["freq"])[:, None].expand(-1, c["heads"], -1)
        return {"q_nope": q[..., :dn].contiguous(), "q_rope": _exact_turn(q[..., dn:].contiguous(), angles.contiguous(), s["gain"], c["half"])}
    dc = c["d_c"]
    x = s["rows"].double().flatten(0, 1)
    angles = s["positions"].double().flatten()[:, None] * s["freq"]
    latent = x[:, :dc]
    if c["norm"]:
        latent = latent / (latent.square().sum(1, keepdim=True) / dc + s["eps"]).sqrt() * s["weight"].double()
    row = torch.cat((latent, _exact_turn(x[:, dc:].contiguous(), angles, s["gain"], c["half"])), 1)
    at = _slots(s)
    kv = torch.zeros(s["kv"].shape, dtype=torch.float64, device=DEV)
    kv_scale = None
    if c["cache"] == "fp8":
        scale = row.abs().max(1).values / E4M3_MAX
        row = row / scale[:, None]
        kv_scale = torch.zeros(s["kv_scale"].shape, dtype=torch.float64, device=DEV)
        kv_scale.view(-1).index_copy_(0, at, scale)
    kv.view(-1, row.shape[1]).index_copy_(0, at, row)
    return {"kv": kv, "kv_scale": kv_scale}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    kind = c["kind"]
    if kind in ("norm", "quant"):
        n, b = c["tokens"] * c["dim"], _BYTES[c["io"]]
        codes = n + 4 * c["tokens"] * _blocks(c["dim"]) if kind == "quant" or c["codes"] else 0
        if kind == "quant":
            return {"bytes": n * b + codes, "flops": 3 * n}
        return {"bytes": n * b * (1 + 2 * c["residual"] + c["plain"]) + c["dim"] * b + codes, "flops": 7 * n}
    if kind == "gemm":
        m, n, k = c["tokens"], c["n"], c["k"]
        return {"bytes": m * k + n * k + 4 * _blocks(k) * (m + _blocks(n)) + m * n * _BYTES[c["out"]], "flops": 2 * m * n * k}
    if kind == "rope":
        n = c["tokens"] * c["heads"]
        return {"bytes": 2 * n * (c["d_nope"] + c["d_rope"]) * _BYTES[c["io"]] + 4 * c["tokens"], "flops": 3 * n * c["d_rope"]}
    n, row = c["batch"] * c["new"], c["d_c"] + D_ROPE
    return {"bytes": n * (row * (_BYTES[c["io"]] + _BYTES[c["cache"]]) + 8 + 4 * (c["cache"] == "fp8")),
            "flops": n * (4 * c["d_c"] * c["norm"] + 3 * D_ROPE)}
