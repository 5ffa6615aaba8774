"""fp64 CPU oracle of the differential encoder layers: rotary positions, differential attention, the
norm - gate - residual step, and the encoder made of them.  Written from the definitions, no code shared
with the HIP path.

Readings (the detector's paper has plain layers; these are the library's own):
  - a differential head uses two neighbouring query / key heads and the values in the columns of both;
  - a token's position is (row, column) of its cell's centre in cells of the finest level;
  - the norm of a head's row is a root-mean-square norm with a gain shared by the heads;
  - a frame without keys gives rows of zeros.
"""
import math
from typing import Dict, Optional, Sequence

import numpy as np

from oracle.cfdetr_oracle import LN_EPS, embed_frame, gelu, layer_norm, softmax_rows


def rotary_frequencies(rot_dim: int, n_axes: int = 1, base: float = 10000.0, factor: float = 1.0,
                       trained_len: float = 0.0, keep_turns: float = 32.0, stretch_turns: float = 1.0) -> np.ndarray:
    """Radians per unit of position of the rot_dim / 2 pairs of a head; the axes have equal sets."""
    per_axis = rot_dim // 2 // n_axes
    f = np.tile(base ** -(np.arange(per_axis) / per_axis), n_axes)
    if trained_len == 0.0:
        return f / factor
    keep = np.clip((trained_len * f / (2 * math.pi) - stretch_turns) / (keep_turns - stretch_turns), 0.0, 1.0)
    return f * keep + f / factor * (1.0 - keep)


def rotary(x: np.ndarray, pos: np.ndarray, freq: np.ndarray, heads: int, interleaved: bool) -> np.ndarray:
    """x [M, heads * dh], pos [M, n_axes], freq [n]: every pair turned by its angle."""
    M, d = x.shape
    n, n_axes = len(freq), pos.shape[1]
    out = x.astype(np.float64).reshape(M, heads, d // heads).copy()
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = pos[:, i // (n // n_axes)].astype(np.float64) * freq[i]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        u, v = out[:, :, a].copy(), out[:, :, b].copy()
        out[:, :, a], out[:, :, b] = u * c - v * s, u * s + v * c
    return out.reshape(M, d)


def rms_norm(x: np.ndarray, g: np.ndarray, eps: float = LN_EPS) -> np.ndarray:
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * g.astype(np.float64)


def diff_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, n_heads: int, lam: np.ndarray,
                   head_g: Optional[np.ndarray] = None, scale: Optional[float] = None,
                   key_mask: Optional[np.ndarray] = None) -> np.ndarray:
    """One frame: q [Tq, d], k and v [Tk, d]; n_heads query / key heads, n_heads / 2 differential ones."""
    Tq, d = q.shape
    dh = d // n_heads
    if scale is None:
        scale = dh ** -0.5
    keys = np.arange(k.shape[0]) if key_mask is None else np.flatnonzero(key_mask)
    out = np.zeros((Tq, d))
    if len(keys) == 0:
        return out
    k, v = k[keys].astype(np.float64), v[keys].astype(np.float64)
    for h in range(n_heads // 2):
        first, second = slice(2 * h * dh, (2 * h + 1) * dh), slice((2 * h + 1) * dh, (2 * h + 2) * dh)
        cols = slice(2 * h * dh, (2 * h + 2) * dh)
        a1 = softmax_rows(scale * (q[:, first].astype(np.float64) @ k[:, first].T))
        a2 = softmax_rows(scale * (q[:, second].astype(np.float64) @ k[:, second].T))
        o = (a1 - float(lam[h]) * a2) @ v[:, cols]
        out[:, cols] = o if head_g is None else rms_norm(o, head_g)
    return out


def norm_residual(x: np.ndarray, block: np.ndarray, post=None, gate=None, res_scale: float = 1.0, pre=None):
    """post, pre: functions of rows or None; returns (x', pre(x') or None)."""
    y = block.astype(np.float64)
    if post is not None:
        y = post(y)
    if gate is not None:
        y = gate.astype(np.float64) * y
    new = res_scale * x.astype(np.float64) + y
    return new, None if pre is None else pre(new)


def cell_positions(tok: np.ndarray, n_levels: int) -> np.ndarray:
    """tok [T, 3] = (level, row, column) -> [T, 2]."""
    size = 2.0 ** (n_levels - 1 - tok[:, 0])
    return np.stack([(tok[:, 1] + 0.5) * size, (tok[:, 2] + 0.5) * size], axis=1)


def encode_sequence(x: np.ndarray, pos: np.ndarray, weights: Dict[str, np.ndarray], diff: Dict[str, np.ndarray], n_heads: int,
                    freq: np.ndarray, interleaved: bool = False, res_scale: float = 1.0) -> np.ndarray:
    """Layers of the differential form and the final LayerNorm over one frame's tokens."""
    w, d = weights, x.shape[1]
    f64 = lambda a: np.asarray(a, dtype=np.float64)
    row = lambda name, l: diff[name][l] if name in diff else None
    for l in range(w["w_qkv"].shape[0]):
        a = layer_norm(x, w["ln1_g"][l], w["ln1_b"][l])
        qkv = a @ f64(w["w_qkv"][l]).T + f64(w["b_qkv"][l])
        q, k = (rotary(qkv[:, i * d:(i + 1) * d], pos, freq, n_heads, interleaved) for i in (0, 1))
        o = diff_attention(q, k, qkv[:, 2 * d:], n_heads, diff["lambda"][l], row("head_g", l))
        t = o @ f64(w["w_o"][l]).T + f64(w["b_o"][l])
        post = (lambda y, l=l: rms_norm(y, diff["post1_g"][l])) if "post1_g" in diff else None
        x, m = norm_residual(x, t, post, row("gate1", l), res_scale, lambda y, l=l: layer_norm(y, w["ln2_g"][l], w["ln2_b"][l]))
        t = gelu(m @ f64(w["w_ff1"][l]).T + f64(w["b_ff1"][l])) @ f64(w["w_ff2"][l]).T + f64(w["b_ff2"][l])
        post = (lambda y, l=l: rms_norm(y, diff["post2_g"][l])) if "post2_g" in diff else None
        x, _ = norm_residual(x, t, post, row("gate2", l), res_scale)
    return layer_norm(x, w["lnf_g"], w["lnf_b"])


def fine_encode(images: np.ndarray, tok: np.ndarray, cu_seqlens: np.ndarray, patch: Sequence[int], weights, diff, n_heads: int,
                freq: np.ndarray, interleaved: bool = False, res_scale: float = 1.0) -> np.ndarray:
    """Every frame on its own token set (also the coarse pass, on the coarse grid's tokens)."""
    ys = []
    for i in range(images.shape[0]):
        lo, hi = int(cu_seqlens[i]), int(cu_seqlens[i + 1])
        if hi > lo:
            x = embed_frame(images[i], tok[lo:hi], patch, weights)
            ys.append(encode_sequence(x, cell_positions(tok[lo:hi], len(patch)), weights, diff, n_heads, freq, interleaved, res_scale))
    return np.concatenate(ys)
