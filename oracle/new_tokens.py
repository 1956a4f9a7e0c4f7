"""Rotary positions and the cache of 8 bits, in fp64 numpy, written from their formulas."""
from __future__ import annotations

import math

import numpy as np

from .bf16 import bf16_bits_to_f64, f64_to_bf16_bits


def rope_frequencies(rot: int, base: float, factor: float = 1.0, low_turns: float = 0.0, high_turns: float = 0.0,
                     original_len: float = 0.0) -> np.ndarray:
    """f_i = base^(-2i / rot), scaled: all divided by `factor`, or, with original_len, by the turns a pair makes within it."""
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if original_len <= 0:
        return f / factor
    out = []
    for x in f:
        turns = original_len * x / (2 * math.pi)
        if turns <= low_turns:
            out.append(x / factor)
        elif turns >= high_turns:
            out.append(x)
        else:
            w = (turns - low_turns) / (high_turns - low_turns)
            out.append((1 - w) * x / factor + w * x)
    return np.array(out)


def rope_turn(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, interleaved: bool) -> np.ndarray:
    """x f64 [..., D]; cos, sin f64 [..., rot / 2] (broadcast).  Unrounded."""
    half = cos.shape[-1]
    y = np.array(x, dtype=np.float64)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[..., a] = x[..., a] * cos[..., i] - x[..., b] * sin[..., i]
        y[..., b] = x[..., b] * cos[..., i] + x[..., a] * sin[..., i]
    return y


def e4m3_values() -> np.ndarray:
    """What the 128 non-negative codes of e4m3 stand for (the last one is NaN)."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


def nearest_value(x: np.ndarray, fmt: str) -> np.ndarray:
    """The nearest value of the format, ties to the even code (e4m3) or number (int8); |x| within its range."""
    if fmt == "int8":
        return np.rint(x) + 0.0                                                  # (whole numbers have one zero)
    v = e4m3_values()
    a = np.abs(x)
    hi = np.clip(np.searchsorted(v, a), 0, len(v) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = v[hi] - a, a - v[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0)) | (v[hi] == a)
    return np.copysign(np.where(take_hi, v[hi], v[lo]), x)


def quantise_block(x: np.ndarray, fmt: str):
    """(values before the scale, scale) of one block [rows, D] in f64; a block with an infinity or a NaN: zeros, NaN."""
    most = 448.0 if fmt == "e4m3" else 127.0
    if not np.isfinite(x).all():
        return np.zeros_like(x), math.nan
    top = np.abs(x).max()
    if top == 0:
        return np.zeros_like(x), 1.0
    e = -126
    while top > most * 2.0 ** e:
        e += 1
    return nearest_value(x / 2.0 ** e, fmt), 2.0 ** e


class Cache8:
    """One (sequence, KV head) of a cache of 8 bits, keys or values, fed row by row."""

    def __init__(self, block: int, fmt: str):
        self.block, self.fmt, self.values, self.scales, self.tail = block, fmt, [], [], []

    def append(self, row_bits: np.ndarray) -> None:
        self.tail.append(bf16_bits_to_f64(row_bits))
        if len(self.tail) == self.block:
            v, s = quantise_block(np.stack(self.tail), self.fmt)
            self.values.append(v)
            self.scales.append(s)
            self.tail = []

    def rows(self) -> np.ndarray:
        """What the cache stands for, f64 [rows, D]."""
        parts = [v * s for v, s in zip(self.values, self.scales)]
        if self.tail:
            parts.append(np.stack(self.tail))
        return np.concatenate(parts) if parts else np.zeros((0, 128))


def attn8(q_bits: np.ndarray, k_rows: np.ndarray, v_rows: np.ndarray, scale: float):
    """One query row over what a cache stands for, f64: (out, weights, lse)."""
    if not len(k_rows):
        return np.zeros(q_bits.shape[-1]), np.zeros(0), -math.inf
    s = scale * (k_rows @ bf16_bits_to_f64(q_bits))
    m = s.max()
    p = np.exp(s - m)
    return (p / p.sum()) @ v_rows, p / p.sum(), m + math.log(p.sum())


def prompt_attn(q: np.ndarray, K: np.ndarray, V: np.ndarray, pos: int, first: int, end: int, scale: float, cap: float = 0.0,
                slope: float = 0.0):
    """One query row (position `pos`) over rows first .. end - 1 of K, V (f64 [rows, D]): (out, lse); no row: (0, -inf)."""
    j = np.arange(max(first, 0), min(end, len(K)))
    if not len(j):
        return np.zeros(q.shape[-1]), -math.inf
    s = scale * (K[j] @ q)
    if cap > 0:
        s = cap * np.tanh(s / cap)
    s = s - slope * np.abs(pos - j)
    m = s.max()
    p = np.exp(s - m)
    return (p / p.sum()) @ V[j], m + math.log(p.sum())


__all__ = ["rope_frequencies", "rope_turn", "e4m3_values", "nearest_value", "quantise_block", "Cache8", "attn8", "prompt_attn",
           "bf16_bits_to_f64", "f64_to_bf16_bits"]
