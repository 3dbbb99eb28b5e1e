"""Plain reference of the mixed cache's content and of the rotary positions:
numpy in 64 bits, from the definitions alone.  The attention and its bounds are
latent_ref's: keys and values of a sequence, which of them a row sees.

LOW elements are code * scale in 64 bits.  Their weights and values are rounded
to fp16 (2^-11 each), within the bf16 step (2^-8) that the bounds count for a
weight.  To an output's bound come
  2^-33 sum |v|  fp16's smallest step is 2^-24, a weight's rounding 2^-25 at
                 least, and the largest weight of a row (of a piece of its keys)
                 2^8 or more, as the reference lies 8 under a maximum: an entry's
                 weight lacks 2^-33 of the largest at most, and the sum that
                 divides it is no less than the largest
  2^-20          where a value is above 19,096 (a scale above 2728): the values of
                 its page are taken at 1 / 32, where fp16 rounds by 2^-25 at least

Rotary bounds: an element x cos a - y sin a is off by half a step of bf16
(2^-8 of it) and by (|x| + |y|) m times
  2^-21.3  the angle: the turns' 64-bit product, 2^-24 turns at position 2^31
  2^-22.3  the reduced turns rounded to fp32, half a turn at most
  2^-22    sine and cosine of fp32 (2 units in the last place), and with m
  2^-23    the two products and their sum
together below 2^-19.9.
"""

from __future__ import annotations

import math

import numpy as np
import torch

from . import latent_ref
from .latent_ref import DROP, HIGH, LOW, U16, f64  # noqa: F401

ROPE_TOL = 2.0 ** -19.9


def low_values(c):
    """code * scale in 64 bits of rows [n, 32 m]."""
    x = c.reshape(len(c), -1, 32)
    s = np.minimum(np.abs(x).max(-1, keepdims=True) / 7.0, 65504.0).astype(np.float16).astype(np.float64)
    return np.where(s > 0, np.clip(np.rint(x / np.where(s > 0, s, 1.0)), -7, 7) * s, 0.0).reshape(c.shape)


class RefCache:
    """What one layer's cache holds: per sequence its tokens' action, key and value by position."""

    def __init__(self, batch, actions, n_sink=0, window=0, max_tokens=1 << 30, n_tags=None):
        self.act, self.n_sink, self.window, self.max_tokens = list(actions), n_sink, window, max_tokens
        self.tokens = [[] for _ in range(batch)]

    def append(self, b, k, v, tags=None, keep_all=False):
        """k, v [n, KV, D] (bf16 values in 64 bits)."""
        for j in range(len(k)):
            pos = len(self.tokens[b])
            if pos >= self.max_tokens:
                break
            tag = 0 if tags is None else int(tags[j])
            forced = keep_all or pos < self.n_sink or tag >= len(self.act)
            self.tokens[b].append((HIGH if forced else self.act[tag], k[j], v[j]))

    def n_pos(self, b):
        return len(self.tokens[b])

    def visible(self, b):
        """(positions [n], keys [n, KV, D], values [n, KV, D]) that the cache holds now."""
        t, n = self.tokens[b], len(self.tokens[b])
        at = [p for p in range(n) if p >= n - self.window or t[p][0] != DROP]
        if not at:
            return np.zeros(0, np.int64), None, None
        k, v = np.stack([t[p][1] for p in at]), np.stack([t[p][2] for p in at])
        coded = np.array([p < n - self.window and t[p][0] == LOW for p in at])
        if coded.any():
            for x in (k, v):
                x[coded] = low_values(x[coded].reshape(int(coded.sum()), -1)).reshape(-1, *x.shape[1:])
        return np.array(at, np.int64), k, v


def prompt(cache, b, q, first, scale):
    """q [n, Hq, D] at positions first ..: out, lse and their bounds, [n, Hq, D] and [n, Hq]."""
    n, hq, d = q.shape
    pos, k, v = cache.visible(b)
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    out_tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
    if len(pos):
        seen = pos[None] <= first + np.arange(n)[:, None]
        for h in range(hq):
            g = h * k.shape[1] // hq
            out[:, h], lse[:, h], out_tol[:, h], lse_tol[:, h] = latent_ref.attention(q[:, h], k[:, g], v[:, g], scale,
                                                                                      seen)
            out_tol[:, h] += 2.0 ** -33 * (seen @ np.abs(v[:, g]))
        out_tol += 2.0 ** -20 * bool((np.abs(v) > 19096).any())
    return out, lse, out_tol, lse_tol


def frequencies(rot_dim, base, scaling="plain", factor=1.0, original=1, low=1.0, high=32.0):
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])
    if scaling == "linear":
        return f / factor
    if scaling == "parts":
        g = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return g * f + (1 - g) * f / factor
    return f


def rotate(x, pos, freq, rot_first, rot_dim, interleaved, magnitude=1.0):
    """x [n, heads, D] in 64 bits at positions pos [n]: the rotated rows and the bound of their elements."""
    i = np.arange(rot_dim // 2)
    one, two = (rot_first + 2 * i, rot_first + 2 * i + 1) if interleaved else (rot_first + i, rot_first + rot_dim // 2 + i)
    # the angle in turns of 64 bits loses what 2 pi p f loses: reduce p f / (2 pi) exactly as far as 64 bits go
    t = pos[:, None].astype(np.longdouble) * (freq / (2 * np.pi))[None].astype(np.longdouble)
    a = ((t - np.rint(t)) * 2 * np.longdouble(np.pi)).astype(np.float64)[:, None]
    y, tol = x.copy(), np.zeros_like(x)
    u, w = x[:, :, one], x[:, :, two]
    y[:, :, one], y[:, :, two] = magnitude * (u * np.cos(a) - w * np.sin(a)), magnitude * (u * np.sin(a) + w * np.cos(a))
    size = abs(magnitude) * (np.abs(u) + np.abs(w)) * ROPE_TOL
    tol[:, :, one] = U16 * np.abs(y[:, :, one]) + size
    tol[:, :, two] = U16 * np.abs(y[:, :, two]) + size
    return y, tol
