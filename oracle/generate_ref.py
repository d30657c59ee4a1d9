"""Generation operators -- CPU oracle, TEST INFRASTRUCTURE ONLY.

The 8-bit cache, the attention over it and beam search's selection, from their definitions: numpy,
fp64, with fp32 where a definition names it (what decides a code is decided in the stated type).
"""
from __future__ import annotations

from typing import List, Optional

import numpy as np

from . import termezo_ref as orc

BLOCK = 64


def to_type(x, bf16: bool) -> np.ndarray:
    x = np.asarray(x, np.float32)
    return orc.bf16_round(x) if bf16 else x


def rotate(x: np.ndarray, pos: np.ndarray, base: float) -> np.ndarray:
    """fp32 rotation of x [T, H, hd] at positions pos: angles in fp64, cosine and sine in fp32."""
    if base == 0.0:
        return np.asarray(x, np.float32)
    half = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None] * base ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(ang).astype(np.float32)[:, None], np.sin(ang).astype(np.float32)[:, None]
    a, b = np.asarray(x[..., :half], np.float32), np.asarray(x[..., half:], np.float32)
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def quantise_block(x: np.ndarray):
    """Codes and step of a block of one head: x [64, hd] fp32 values."""
    if not np.isfinite(x).all():
        return np.zeros(x.shape, np.int32), np.float32(np.nan)
    a = np.float32(max(np.abs(x).max(), np.float32(1e-30)))
    q = np.rint(x * (np.float32(127.0) * (np.float32(1.0) / a))).astype(np.int32)
    return q, a * (np.float32(1.0) / np.float32(127.0))


class Sequence:
    """One layer of one sequence: keys (rotated, in the activation type) and values."""

    def __init__(self, bf16: bool, base: float):
        self.bf16, self.base = bf16, base
        self.k: Optional[np.ndarray] = None
        self.v: Optional[np.ndarray] = None

    def copy(self) -> "Sequence":
        s = Sequence(self.bf16, self.base)
        s.k, s.v = self.k, self.v
        return s

    def __len__(self):
        return 0 if self.k is None else len(self.k)

    def append(self, k, v):
        n = len(self)
        k = to_type(rotate(k, np.arange(n, n + len(k)), self.base), self.bf16)
        v = to_type(v, self.bf16)
        self.k = k if self.k is None else np.concatenate([self.k, k])
        self.v = v if self.v is None else np.concatenate([self.v, v])

    def values(self):
        """What the cache holds, as fp32."""
        out = []
        for x in (self.k, self.v):
            y = x.astype(np.float32).copy()
            for j in range(len(x) // BLOCK):
                for h in range(x.shape[1]):
                    q, d = quantise_block(x[j * BLOCK:(j + 1) * BLOCK, h])
                    y[j * BLOCK:(j + 1) * BLOCK, h] = q.astype(np.float32) * d
            out.append(y)
        return out


def attend(seq: Sequence, q: np.ndarray):
    """Attention of the last len(q) tokens: q [n, H, hd] unrotated.  Returns out [n, H, hd] (fp64),
    sum_t p_t |v_t| and the largest sum_d |q_d k_d| / sqrt(hd) of every query (for error bounds)."""
    n, H, hd = q.shape
    T = len(seq)
    k, v = (x.astype(np.float64) for x in seq.values())
    qr = rotate(q, np.arange(T - n, T), seq.base).astype(np.float64)
    out, mag, big = np.zeros((n, H, hd)), np.zeros((n, H, hd)), np.zeros((n, H, 1))
    late = np.arange(T)[None] > np.arange(T - n, T)[:, None]
    for h in range(H):
        g = h * k.shape[1] // H
        s = np.where(late, -np.inf, qr[:, h] @ k[:, g].T / np.sqrt(hd))
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h] = p @ v[:, g]
        mag[:, h] = p @ np.abs(v[:, g])
        big[:, h, 0] = np.where(late, 0.0, np.abs(qr[:, h]) @ np.abs(k[:, g]).T / np.sqrt(hd)).max(1)
    return out, mag, big


def beam_select(logits, scores, n_out: int, eos: int = -1, finished=None, history=None):
    """Selection for one search: logits [W, V], scores [W].  Returns scores (fp64), tokens, parents,
    finished, history."""
    W, V = logits.shape
    x = np.where(np.isnan(logits), -np.inf, logits).astype(np.float64)
    c = np.full((W, V), -np.inf)
    fin = np.zeros(W, bool) if finished is None else np.asarray(finished, bool)
    for b in range(W):
        if fin[b]:
            c[b, eos] = scores[b]
            continue
        top = x[b].max()
        if not np.isfinite(top):
            continue
        c[b] = float(scores[b]) + x[b] - (top + np.log(np.exp(x[b] - top).sum()))
    c = np.where(np.isnan(c), -np.inf, c).reshape(-1)
    pick = np.lexsort((np.arange(c.size), -c))[:n_out]
    tok, par = pick % V, pick // V
    done = fin[par] | (tok == eos)
    hist = None if history is None else np.concatenate([history[par], tok[:, None]], 1)
    return c[pick], tok, par, done, hist
