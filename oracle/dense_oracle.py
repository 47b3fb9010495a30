"""The dense operators around the block attention in fp64 NumPy, one formula per function, no blocking or fusion.

Rows are tokens.  A vector that changes along the rows is [groups, cols]; row r uses group r // group_rows.
"""
from __future__ import annotations

import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activation(v: np.ndarray, act: str) -> np.ndarray:
    if act == "none":
        return v
    with np.errstate(over="ignore"):
        if act == "silu":
            return v / (1.0 + np.exp(-v))
        if act == "gelu_tanh":
            return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    if act == "gelu":
        return 0.5 * v * _erfc(-v / math.sqrt(2.0))
    raise ValueError(act)


def of_rows(vectors: np.ndarray, rows: int, group_rows: int) -> np.ndarray:
    return vectors[np.arange(rows) // group_rows]


def linear_ref(x, w, bias=None, act="none", gate=None, gate_rows=0, residual=None) -> np.ndarray:
    v = x @ w.T
    if bias is not None:
        v = v + bias
    v = activation(v, act)
    if gate is not None:
        v = v * of_rows(gate, x.shape[0], gate_rows)
    return v if residual is None else v + residual


def norm_ref(v: np.ndarray, kind: str, eps: float) -> np.ndarray:
    """RMS or layer norm over the last axis."""
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        return v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)


def gated_norm_ref(x, y=None, post="none", post_weight=None, gate=None, gate_rows=0, norm="layer", weight=None, bias=None,
                   scale=None, shift=None, mod_rows=0, eps=1e-6):
    """(s, out)"""
    s = x
    if y is not None:
        y = norm_ref(y, post, eps)
        if post_weight is not None:
            y = y * post_weight
        if gate is not None:
            y = y * of_rows(gate, x.shape[0], gate_rows)
        s = x + y
    o = norm_ref(s, norm, eps)
    if weight is not None:
        o = o * weight
    if bias is not None:
        o = o + bias
    if scale is not None:
        o = o * (1.0 + of_rows(scale, x.shape[0], mod_rows))
    if shift is not None:
        o = o + of_rows(shift, x.shape[0], mod_rows)
    return s, o


def qk_norm_rope_ref(x, weight, scope, eps, grid, frame_offset, table, tab_frames) -> np.ndarray:
    """rope(rms(x) * weight) of [tokens, heads, dim]; `table` is the fp32 (cos, sin) table of the rotary embedding."""
    tokens, heads, dim = x.shape
    frames, grid_h, grid_w = grid
    if scope == "row":
        v = norm_ref(x.reshape(tokens, heads * dim), "rms", eps)
        v = (v if weight is None else v * weight).reshape(x.shape)
    else:
        v = norm_ref(x, "rms", eps)
        v = v if weight is None else v * weight
    pairs_hw = dim // 6
    pairs = (dim // 2 - 2 * pairs_hw, pairs_hw, pairs_hw)
    t = np.arange(tokens)
    where = (frame_offset + t // (grid_h * grid_w), t // grid_w % grid_h, t % grid_w)
    parts, at = [], 0
    for count, positions, pos in zip(pairs, (tab_frames, grid_h, grid_w), where):
        parts.append(table[at:at + 2 * count * positions].reshape(positions, count, 2)[pos])
        at += 2 * count * positions
    cs = np.concatenate(parts, 1).astype(np.float64)[:, None]
    z = (v[..., 0::2] + 1j * v[..., 1::2]) * (cs[..., 0] + 1j * cs[..., 1])
    return np.stack([z.real, z.imag], -1).reshape(x.shape)
