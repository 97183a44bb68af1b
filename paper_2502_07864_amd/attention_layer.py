"""One converted attention layer, from hidden states to hidden states.

The calls of ``layer.py`` and ``mla.py`` in the order in which a serving loop makes them:

    rms_norm_fp8 (+ residual)  ->  gemm_fp8: queries, cache rows  ->  rope_queries, cache_store
    ->  absorb_q, decode_paged(_multi), merge_out_proj   (or prefill_mha)
    ->  quantize_rows  ->  gemm_fp8: output

Projections run on e4m3 codes, the attention on bf16 queries and the cache as it is stored.  The layer holds its weights
and nothing else: caches, tables and lengths are the caller's, outputs and scratch come from torch's allocator, so that a
step can be captured into a graph.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import layer, mla


class AttentionLayer:
    """W_Q [H * (d_head + d_rope), D] (per head the nope rows, then the rope rows), W_DKVR [d_c + d_rope, D], W_O [D, H *
    d_head] are quantised here, once; W_UK [H, d_head, d_c] and W_UV [H, d_c, d_head] are kept in bf16, norm_weight [D] and
    latent_norm [d_c] (None: the latents are cached as projected) in the type of the hidden states.  rope: (freq, gain) as
    layer.rope_frequencies gives them.  gemm_flags: of the queries' and the output's product (layer.gemm_fp8;
    GEMM_FAST_SUMS: both results are rounded to bf16 anyway); the cache rows, in fp32, always have full sums.
    latent_eps: of the latents' norm, eps where it is None."""

    def __init__(self, W_Q: torch.Tensor, W_DKVR: torch.Tensor, W_UK: torch.Tensor, W_UV: torch.Tensor, W_O: torch.Tensor,
                 norm_weight: torch.Tensor, rope: Tuple[torch.Tensor, float], softmax_scale: float, eps: float = 1e-6,
                 latent_norm: Optional[torch.Tensor] = None, layout: int = layer.ROPE_INTERLEAVED, gemm_flags: int = 0,
                 latent_eps: Optional[float] = None):
        H, d_head, d_c = W_UK.shape
        self.freq, self.gain = rope
        self.H, self.d_head, self.d_c, self.d_rope = H, d_head, d_c, 2 * self.freq.numel()
        D = norm_weight.numel()
        shapes = {"W_Q": (W_Q, (H * (d_head + self.d_rope), D)), "W_DKVR": (W_DKVR, (d_c + self.d_rope, D)),
                  "W_UV": (W_UV, (H, d_c, d_head)), "W_O": (W_O, (D, H * d_head))}
        for name, (w, shape) in shapes.items():
            if tuple(w.shape) != shape:
                raise ValueError(f"{name} must be {list(shape)}, got {list(w.shape)}")
        if W_UK.dtype != torch.bfloat16 or W_UV.dtype != torch.bfloat16:
            raise TypeError(f"W_UK and W_UV must be bfloat16, got {W_UK.dtype} and {W_UV.dtype}")
        if D % 16 or (H * d_head) % 16:
            raise ValueError("the model dimension and H * d_head must be multiples of 16")
        self.W_Q, self.W_DKVR, self.W_O = (layer.quantize_weights(w.contiguous()) for w in (W_Q, W_DKVR, W_O))
        self.W_UK, self.W_UV = W_UK.contiguous(), W_UV.contiguous()
        self.norm_weight = norm_weight
        # the cache rows come out of their product in fp32, to be rounded once where they are stored
        self.latent_norm = None if latent_norm is None else latent_norm.float()
        self.latent_eps = float(eps if latent_eps is None else latent_eps)
        self.softmax_scale, self.eps, self.layout, self.gemm_flags = float(softmax_scale), float(eps), int(layout), int(gemm_flags)

    @classmethod
    def from_conversion(cls, cv: dict, W_Q: torch.Tensor, W_O: torch.Tensor, norm_weight: torch.Tensor, d_head: int,
                        rope: Tuple[torch.Tensor, float], **kw) -> "AttentionLayer":
        """The layer that convert.convert_layer's outputs stand for, with the query and output projections of the layer
        that was converted (W_Q [h * d, D], W_O [D, h * d]): head i's rope rows are W_QR[i] W_Q_i, in interleaved pairs.

        rope: its d_rope / 2 = keep * d / (2 M) frequencies, of the converted layer's base.  Pair G * keep + r belongs to
        FreqFold group G, so for any keep it may turn with the group's first frequency:
            freq, gain = layer.rope_frequencies(d // M, base);  rope = (freq.repeat_interleave(keep), gain)
        which is rope_frequencies(d_rope, base) for keep = 1.  For keep = M rope_frequencies(d, base) gives each pair one of
        its group's own M frequencies, and the layer's own for M = 1.  For 1 < keep < M rope_frequencies(d_rope, base) is
        neither."""
        if kw.get("layout", layer.ROPE_INTERLEAVED) != layer.ROPE_INTERLEAVED:
            raise ValueError("the conversion's rope rows are interleaved pairs")
        h, d_rope, d = cv["W_QR"].shape
        D = W_Q.shape[1]
        per_head = W_Q.double().view(h, d, D)
        rows = torch.cat((per_head, torch.bmm(cv["W_QR"].double(), per_head)), 1).view(h * (d + d_rope), D)
        bf = torch.bfloat16
        # (the quantised ones in fp32: a rounding to bf16 before the codes' own would move values between two of them)
        return cls(rows.float(), torch.cat((cv["W_DKV"], cv["W_KR"]), 0).float(), cv["W_UK"].to(bf), cv["W_UV"].to(bf), W_O.float(),
                   norm_weight, rope, d_head ** -0.5, **kw)

    def _before(self, x, residual, positions, kv_cache, page_table, kv_scale):
        """Norm, projections, rotation and the new cache rows.  x [B, q_len, D], positions [B, q_len]."""
        B, T, D = x.shape
        codes, scales, s, _ = layer.rms_norm_fp8(x.view(B * T, D), self.norm_weight, self.eps,
                                                 residual=None if residual is None else residual.view(B * T, D))
        rows = layer.gemm_fp8(codes, scales, *self.W_DKVR, dtype=torch.float32)
        layer.cache_store(rows.view(B, T, -1), positions, self.freq, kv_cache, page_table, self.d_c, self.gain, self.layout,
                          self.latent_norm, self.latent_eps, kv_scale)
        q = layer.gemm_fp8(codes, scales, *self.W_Q, flags=self.gemm_flags)
        q_nope, q_rope = layer.rope_queries(q.view(B * T, self.H, -1), positions.view(B * T), self.freq, self.gain, self.layout)
        return q_nope, q_rope, (x if s is None else s).view(B, T, D)

    def _after(self, out, B, T):
        """Output projection of the heads' results [B, T, H, d_head]."""
        codes, scales = layer.quantize_rows(out.view(B * T, self.H * self.d_head))
        return layer.gemm_fp8(codes, scales, *self.W_O, flags=self.gemm_flags).view(B, T, -1)

    def decode(self, x: torch.Tensor, positions: torch.Tensor, kv_cache: torch.Tensor, page_table: torch.Tensor,
               seq_lens: torch.Tensor, residual: Optional[torch.Tensor] = None, kv_scale: Optional[torch.Tensor] = None,
               num_splits: int = 16) -> Tuple[torch.Tensor, torch.Tensor]:
        """The newest tokens of every sequence (one, or a few drafted ones): their rows join the cache, then they attend to
        it.  x and residual [B, q_len, D] bf16, positions [B, q_len] int32 = seq_len - q_len + i, seq_lens [B] int32 with the
        new tokens counted, kv_cache bf16 or fp8 (with kv_scale).  Returns (output [B, q_len, D], residual' = x + residual),
        the next layer's x and residual."""
        B, T, _ = x.shape
        q_nope, q_rope, s = self._before(x, residual, positions, kv_cache, page_table, kv_scale)
        q_abs = mla.absorb_q(q_nope, self.W_UK)
        shape = (B, T, self.H, -1)
        ws = mla.decode_paged_multi(q_abs.view(shape), q_rope.view(shape), kv_cache, page_table, seq_lens, self.softmax_scale,
                                    num_splits=num_splits, kv_scale=kv_scale, flags=mla.FLAG_SKIP_MERGE)
        _, out = mla.merge_out_proj_multi(ws, self.W_UV, B, T, num_splits)
        return self._after(out, B, T), s

    def prefill(self, x: torch.Tensor, positions: torch.Tensor, kv_cache: torch.Tensor, page_table: torch.Tensor,
                seq_lens: torch.Tensor, residual: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The same for whole prompts or chunks of them on a bf16 cache with pages of 64 rows: keys and values are
        materialised per head (mla.prefill_mha)."""
        B, T, _ = x.shape
        q_nope, q_rope, s = self._before(x, residual, positions, kv_cache, page_table, None)
        shape = (B, T, self.H, -1)
        out = mla.prefill_mha(q_nope.view(shape), q_rope.view(shape), self.W_UK, self.W_UV, kv_cache, page_table, seq_lens,
                              self.softmax_scale)
        return self._after(out, B, T), s
