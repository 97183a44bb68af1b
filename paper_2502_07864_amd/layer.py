"""Python binding of the operators around the attention (``include/mla_layer_gfx950.h``): RMS norm with the
residual's addition and 8-bit output, projections on 8-bit codes, the queries' rotation, cache rows of new tokens.

Argument marshalling only, as in ``mla.py``: torch tensors on the GPU in, device pointers and the current HIP stream
to the C entry point of the same name, output tensors out.  Outputs that are passed in are written in place, densely from
their first element on (no allocation; their type and room are checked, their shape is the caller's); the others are
allocated.  There is no fallback path.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import mla
from .mla import _cache_code, _check, _dev, _io_code, _room, _stream, lib

ROPE_INTERLEAVED, ROPE_HALF = 0, 1
GEMM_FAST_SUMS = 1
_KINDS = {"none": 0, "linear": 1, "yarn": 2}
_CODES = (torch.float8_e4m3fn, torch.uint8)


def _blocks(n: int) -> int:
    return -(-n // 128)


def _rows(x: torch.Tensor, name: str, T: int, width: int):
    """(pointer, pitch) of T rows of `width` elements, each dense, at equal distances."""
    if not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError(f"{name} must have dense rows")
    pitch = x.stride(0) if T > 1 else width
    if pitch < width:
        raise ValueError(f"the rows of {name} overlap")
    return x.data_ptr(), pitch


def _like(t: Optional[torch.Tensor], x: torch.Tensor, shape, name: str):
    """A dense operand of x's type."""
    if t is not None and (t.dtype != x.dtype or tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} must be {list(shape)} of {x.dtype}")
    return _dev(t, name)


def _typed(t: Optional[torch.Tensor], x: torch.Tensor, name: str):
    """An output of x's type."""
    if t is not None and t.dtype != x.dtype:
        raise TypeError(f"{name} must be {x.dtype}, got {t.dtype}")
    return _dev(t, name)


def _new_codes(T: int, D: int, device, codes, scales):
    if codes is None:
        codes = torch.empty((T, D), dtype=torch.float8_e4m3fn, device=device)
    if scales is None:
        scales = torch.empty((_blocks(D), T), dtype=torch.float32, device=device)
    if codes.dtype not in _CODES or scales.dtype != torch.float32:
        raise TypeError("codes must be float8_e4m3fn or uint8, scales float32")
    return codes, scales


# As in mla.py the native path is asked first, and what it does not take (None) the checks below decide.

def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
             residual: Optional[torch.Tensor] = None, residual_out: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """y = s / sqrt(mean(s^2) + eps) * weight with s = x + residual;  x [T, D] (rows may be apart), residual [T, D],
    weight [D].  Returns (y, s), s None without a residual."""
    fast = mla._fast
    if fast is not None and out is not None:
        status = fast.rms_norm(x, weight, eps, residual, residual_out, out, None, None)
        if status == 0:
            return out, residual_out
        if status is not None:
            _check(status, "mla_rms_norm")
    if out is None:
        if x.dim() != 2:
            raise ValueError("x must be [T, D]")
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    return _norm(x, weight, eps, residual, residual_out, out, None, None)[2:][::-1]


def rms_norm_fp8(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 residual: Optional[torch.Tensor] = None, codes: Optional[torch.Tensor] = None,
                 scales: Optional[torch.Tensor] = None, residual_out: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None):
    """rms_norm whose y comes as e4m3 codes [T, D] and scales [ceil(D/128), T], for gemm_fp8.
    Returns (codes, scales, s, y): s None without a residual, y None unless `out` is passed (it is then written too)."""
    fast = mla._fast
    if fast is not None and codes is not None:
        status = fast.rms_norm(x, weight, eps, residual, residual_out, out, codes, scales)
        if status == 0:
            return codes, scales, residual_out, out
        if status is not None:
            _check(status, "mla_rms_norm")
    if codes is None or scales is None:
        if x.dim() != 2:
            raise ValueError("x must be [T, D]")
        codes, scales = _new_codes(*x.shape, x.device, codes, scales)
    return _norm(x, weight, eps, residual, residual_out, out, codes, scales)


def _norm(x, weight, eps, residual, residual_out, out, codes, scales):
    if x.dim() != 2:
        raise ValueError("x must be [T, D]")
    if residual is None and residual_out is not None:
        raise ValueError("residual_out without a residual")
    if residual is not None and residual_out is None:
        residual_out = torch.empty_like(residual, memory_format=torch.contiguous_format)
    T, D = x.shape
    px, pitch = _rows(x, "x", T, D)
    if codes is not None:
        _new_codes(T, D, x.device, codes, scales)
    args = (px, _like(residual, x, (T, D), "residual"), _like(weight, x, (D,), "weight"), _typed(residual_out, x, "residual_out"),
            _typed(out, x, "out"), _dev(codes, "codes"), _dev(scales, "scales"), T, D, pitch, float(eps), _io_code(x), _stream(x))
    _room(residual_out, T * D, x.element_size(), "residual_out")
    _room(out, T * D, x.element_size(), "out")
    _room(codes, T * D, 1, "codes")
    _room(scales, T * _blocks(D), 4, "scales")
    _check(lib().mla_rms_norm(*args), "mla_rms_norm")
    return codes, scales, residual_out, out


def quantize_rows(x: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None):
    """e4m3 codes [T, D] and scales [ceil(D/128), T] of x [T, D] (rows may be apart).  Returns (codes, scales)."""
    fast = mla._fast
    if fast is not None and codes is not None:
        status = fast.quantize_rows(x, codes, scales)
        if status == 0:
            return codes, scales
        if status is not None:
            _check(status, "mla_quantize_rows")
    if x.dim() != 2:
        raise ValueError("x must be [T, D]")
    T, D = x.shape
    px, pitch = _rows(x, "x", T, D)
    codes, scales = _new_codes(T, D, x.device, codes, scales)
    args = (px, _dev(codes, "codes"), _dev(scales, "scales"), T, D, pitch, _io_code(x), _stream(x))
    _room(codes, T * D, 1, "codes")
    _room(scales, T * _blocks(D), 4, "scales")
    _check(lib().mla_quantize_rows(*args), "mla_quantize_rows")
    return codes, scales


def quantize_weights(w: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None):
    """e4m3 codes [N, K] and scales [ceil(N/128), ceil(K/128)] of w [N, K].  Returns (codes, scales)."""
    if w.dim() != 2:
        raise ValueError("w must be [N, K]")
    N, K = w.shape
    if codes is None:
        codes = torch.empty((N, K), dtype=torch.float8_e4m3fn, device=w.device)
    if scales is None:
        scales = torch.empty((_blocks(N), _blocks(K)), dtype=torch.float32, device=w.device)
    if codes.dtype not in _CODES or scales.dtype != torch.float32:
        raise TypeError("codes must be float8_e4m3fn or uint8, scales float32")
    args = (_dev(w, "w"), _dev(codes, "codes"), _dev(scales, "scales"), N, K, _io_code(w), _stream(w))
    _room(codes, N * K, 1, "codes")
    _room(scales, _blocks(N) * _blocks(K), 4, "scales")
    _check(lib().mla_quantize_weights(*args), "mla_quantize_weights")
    return codes, scales


def gemm_fp8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().mla_gemm_fp8_workspace_bytes(M, N, K))


def gemm_fp8(a: torch.Tensor, a_scales: torch.Tensor, w: torch.Tensor, w_scales: torch.Tensor,
             out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             dtype: torch.dtype = torch.bfloat16, flags: int = 0) -> torch.Tensor:
    """out [M, N] = (a * a_scales) (w * w_scales)^T;  a [M, K] and w [N, K] e4m3 codes, a_scales [ceil(K/128), M],
    w_scales [ceil(N/128), ceil(K/128)].  out float32 or bfloat16 (`dtype` where it is allocated here).
    flags GEMM_FAST_SUMS: the matrix cores may add the 8-bit products as they are (up to twice the rate; results 1.5e-5
    off for random operands, at most 7 * 2^-13 of the sum of the products' magnitudes)."""
    fast = mla._fast
    if fast is not None and out is not None:
        status = fast.gemm_fp8(a, a_scales, w, w_scales, out, workspace, flags)
        if status == 0:
            return out
        if status is not None and not (status == -4 and workspace is None):      # (sizes that want scratch: allocated below)
            _check(status, "mla_gemm_fp8")
    if a.dim() != 2 or w.dim() != 2 or a.shape[1] != w.shape[1]:
        raise ValueError("a must be [M, K] and w [N, K]")
    if a.dtype not in _CODES or w.dtype not in _CODES:
        raise TypeError("a and w must be float8_e4m3fn or uint8")
    (M, K), N = a.shape, w.shape[0]
    if a_scales.dtype != torch.float32 or w_scales.dtype != torch.float32:
        raise TypeError("scales must be float32")
    if tuple(a_scales.shape) != (_blocks(K), M) or tuple(w_scales.shape) != (_blocks(N), _blocks(K)):
        raise ValueError("a_scales must be [ceil(K/128), M], w_scales [ceil(N/128), ceil(K/128)]")
    if out is None:
        out = torch.empty((M, N), dtype=dtype, device=a.device)
    if workspace is None:
        workspace = torch.empty(max(16, gemm_fp8_workspace_bytes(M, N, K)), dtype=torch.uint8, device=a.device)
    args = (_dev(a, "a"), _dev(a_scales, "a_scales"), _dev(w, "w"), _dev(w_scales, "w_scales"), _dev(out, "out"),
            _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), M, N, K, _io_code(out),
            int(flags), _stream(a))
    _room(out, M * N, out.element_size(), "out")
    _check(lib().mla_gemm_fp8(*args), "mla_gemm_fp8")
    return out


def rope_frequencies(d_rope: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original: int = 4096,
                     beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda") -> Tuple[torch.Tensor, float]:
    """(freq, gain) for rope_queries and cache_store: radians per position of every pair, fp64 [d_rope / 2] on the
    device, made once per model.  scaling: "none", "linear" (all divided by factor) or "yarn" (pairs that turn often
    within `original` positions kept, slow ones divided, a ramp between; gain 0.1 ln(factor) + 1)."""
    if scaling not in _KINDS:
        raise ValueError(f"scaling must be one of {sorted(_KINDS)}")
    host = torch.empty(max(int(d_rope), 2) // 2, dtype=torch.float64)
    gain = ctypes.c_float()
    _check(lib().mla_rope_frequencies(host.data_ptr(), ctypes.addressof(gain), int(d_rope), float(base), _KINDS[scaling],
                                      float(factor), int(original), float(beta_fast), float(beta_slow)), "mla_rope_frequencies")
    return host.to(device), float(gain.value)


def rope_queries(q: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, gain: float = 1.0,
                 layout: int = ROPE_INTERLEAVED, q_nope: Optional[torch.Tensor] = None,
                 q_rope: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """q [T, H, d_nope + d_rope] (tokens may be apart) -> (q_nope [T, H, d_nope], q_rope [T, H, d_rope]), the rope part
    turned by positions[t] * freq;  positions [T] int32, freq [d_rope / 2] float64 (rope_frequencies)."""
    fast = mla._fast
    if fast is not None and q_rope is not None:
        status = fast.rope_queries(q, positions, freq, gain, layout, q_nope, q_rope)
        if status == 0:
            return q_nope, q_rope
        if status is not None:
            _check(status, "mla_rope_queries")
    if q.dim() != 3:
        raise ValueError("q must be [T, H, d_nope + d_rope]")
    T, H, width = q.shape
    if freq.dtype != torch.float64 or positions.dtype != torch.int32:
        raise TypeError("freq must be float64, positions int32")
    d_rope = 2 * freq.numel()
    d_nope = width - d_rope
    if freq.dim() != 1 or d_nope < 0 or positions.shape != (T,):
        raise ValueError("freq must be [d_rope / 2] with d_rope <= the head's width, positions [T]")
    if H > 1 and q.stride(1) != width:
        raise ValueError("the heads of q must be dense")
    pq, pitch = _rows(q, "q", T, H * width)
    if q_nope is None:
        q_nope = torch.empty((T, H, d_nope), dtype=q.dtype, device=q.device)
    if q_rope is None:
        q_rope = torch.empty((T, H, d_rope), dtype=q.dtype, device=q.device)
    args = (pq, _dev(positions, "positions"), _dev(freq, "freq"), _typed(q_nope, q, "q_nope"), _typed(q_rope, q, "q_rope"), T, H, d_nope,
            d_rope, pitch, float(gain), int(layout), _io_code(q), _stream(q))
    _room(q_nope, T * H * d_nope, q.element_size(), "q_nope")
    _room(q_rope, T * H * d_rope, q.element_size(), "q_rope")
    _check(lib().mla_rope_queries(*args), "mla_rope_queries")
    return q_nope, q_rope


def cache_store(rows: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, kv_cache: torch.Tensor,
                page_table: torch.Tensor, d_c: int, gain: float = 1.0, layout: int = ROPE_INTERLEAVED,
                norm_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                kv_scale: Optional[torch.Tensor] = None) -> None:
    """Writes rows [B, new, d_c + d_rope] (may be apart) into kv_cache at logical positions [B, new]: the latent part
    as it is or RMS-normed with norm_weight [d_c], the rope part turned by positions * freq."""
    fast = mla._fast
    if fast is not None:
        status = fast.cache_store(rows, positions, freq, kv_cache, page_table, d_c, gain, layout, norm_weight, eps, kv_scale)
        if status == 0:
            return
        if status is not None:
            _check(status, "mla_cache_store")
    if rows.dim() != 3 or kv_cache.dim() != 3:
        raise ValueError("rows must be [B, new, d_c + d_rope], kv_cache [num_pages, page_size, d_c + d_rope]")
    B, T, row = rows.shape
    num_pages, page_size, row2 = kv_cache.shape
    if freq.dtype != torch.float64 or positions.dtype != torch.int32 or page_table.dtype != torch.int32:
        raise TypeError("freq must be float64, positions and page_table int32")
    d_rope = row - int(d_c)
    if row2 != row or d_rope < 0 or freq.dim() != 1 or 2 * freq.numel() != d_rope:
        raise ValueError("rows and cache rows must be d_c + d_rope wide, freq [d_rope / 2]")
    if positions.shape != (B, T) or page_table.dim() != 2 or page_table.shape[0] != B:
        raise ValueError("positions must be [B, new], page_table [B, max_pages_per_seq]")
    if B > 1 and T > 1 and rows.stride(0) != T * rows.stride(1):
        raise ValueError("rows must be at equal distances")
    flat = rows[0] if B == 1 else rows[:, 0] if T == 1 else rows
    pitch = rows.stride(1) if B > 1 and T > 1 else flat.stride(0)
    px, pitch = _rows(rows, "rows", 1, row)[0], pitch if B * T > 1 else row
    if kv_scale is not None and (kv_scale.dtype != torch.float32 or tuple(kv_scale.shape) != (num_pages, page_size)):
        raise ValueError("kv_scale must be float32 [num_pages, page_size]")
    args = (px, _dev(positions, "positions"), _dev(freq, "freq"), _like(norm_weight, rows, (int(d_c),), "norm_weight"),
            _dev(kv_cache, "kv_cache"), _dev(kv_scale, "kv_scale"), _dev(page_table, "page_table"), B, T, int(d_c), d_rope, pitch,
            page_size, num_pages, page_table.shape[1], float(gain), int(layout), float(eps), _io_code(rows), _cache_code(kv_cache),
            _stream(rows))
    _check(lib().mla_cache_store(*args), "mla_cache_store")
