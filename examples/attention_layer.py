"""A converted attention layer at work on random weights: prompts through ``prefill``, then decode steps, the step also
from a captured graph.

    python examples/attention_layer.py [--batch 16] [--prompt 1024] [--steps 32] [--cache bf16|fp8] [--full-sums]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

from paper_2502_07864_amd import layer                              # noqa: E402
from paper_2502_07864_amd.attention_layer import AttentionLayer      # noqa: E402

D, H, D_HEAD, D_C, D_ROPE, PAGE = 4096, 32, 128, 512, 64, 64


def random_layer(g: torch.Generator, gemm_flags: int) -> AttentionLayer:
    def w(*shape, fan):
        return (torch.randn(shape, generator=g, device="cuda") * fan ** -0.5).bfloat16()
    return AttentionLayer(
        W_Q=w(H * (D_HEAD + D_ROPE), D, fan=D), W_DKVR=w(D_C + D_ROPE, D, fan=D), W_UK=w(H, D_HEAD, D_C, fan=D_C),
        W_UV=w(H, D_C, D_HEAD, fan=D_C), W_O=w(D, H * D_HEAD, fan=H * D_HEAD), norm_weight=torch.ones(D, device="cuda").bfloat16(),
        rope=layer.rope_frequencies(D_ROPE, scaling="yarn", factor=8.0), softmax_scale=(D_HEAD + D_ROPE) ** -0.5,
        latent_norm=torch.ones(D_C, device="cuda"), gemm_flags=gemm_flags)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--cache", choices=("bf16", "fp8"), default="bf16")
    ap.add_argument("--full-sums", action="store_true", help="the projections' 8-bit products are added without loss (layer.GEMM_FAST_SUMS off)")
    a = ap.parse_args()
    B, L = a.batch, a.prompt
    g = torch.Generator(device="cuda").manual_seed(1)
    lay = random_layer(g, 0 if a.full_sums else layer.GEMM_FAST_SUMS)
    pages = -(-(L + a.steps + 4) // PAGE)
    table = torch.randperm(B * pages, generator=g, device="cuda").to(torch.int32).view(B, pages)
    fp8 = a.cache == "fp8"
    kv = torch.zeros((B * pages, PAGE, D_C + D_ROPE), dtype=torch.float8_e4m3fn if fp8 else torch.bfloat16, device="cuda")
    kv_scale = torch.zeros((B * pages, PAGE), device="cuda") if fp8 else None

    start = torch.arange(L, dtype=torch.int32, device="cuda").repeat(B, 1)
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    x = torch.randn((B, L, D), generator=g, device="cuda").bfloat16()
    if fp8:      # prefill_mha reads bf16 caches: here the prompt goes in as short runs of drafted tokens
        run = 16
        for at in range(0, L, run):
            part = slice(at, min(at + run, L))
            lay.decode(x[:, part].contiguous(), start[:, part].contiguous(), kv, table, torch.full_like(lens, part.stop), kv_scale=kv_scale)
    else:
        lay.prefill(x, start, kv, table, lens)

    hidden, residual = x[:, -1:].contiguous(), torch.zeros((B, 1, D), device="cuda").bfloat16()
    positions = lens.clone().view(B, 1)
    lens = lens + 1

    def step():
        return lay.decode(hidden, positions, kv, table, lens, residual=residual, kv_scale=kv_scale)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, carried = step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        graph.replay()
        hidden.copy_(out)             # (one layer's output stands in for the next token's hidden state)
        positions += 1
        lens += 1
    end.record()
    torch.cuda.synchronize()
    print(f"{B} sequences after prompts of {L}, {a.cache} cache: {begin.elapsed_time(end) / a.steps * 1e3:.1f} us per layer and step, "
          f"|output| {out.float().norm() / out.numel() ** 0.5:.3f} rms, finite: {bool(torch.isfinite(out).all())}")


if __name__ == "__main__":
    main()
