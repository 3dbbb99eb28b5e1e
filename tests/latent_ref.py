"""Plain reference of the latent cache and its attention: numpy in 64 bits,
from the definitions alone, and the tolerances of the tests.

Tolerances are derived, not fitted.  With u16 = 2^-8 (half a step of bf16) and
u32 = 2^-24:
  scores   a dot product of K elements summed in fp32: K u32 sum |q c|, in the
           score's units after the scale, and the scale's and the base change's
           roundings, 4 u32 |s|; call the largest over the entries delta.  A
           weight is then off by a factor e^(2 delta) at most (its own score and
           the maximum's), by its exponential, 2^-22, and by its rounding to
           bf16, u16.
  outputs  |err| <= u16 |o| + (u16 + 2 delta + 2^-22 + n u32) sum p |v|
  lse      |err| <= delta + (n + 16) u32 + 4 u32 |lse|
all times 1.05 for the second-order terms.  Underflow adds 2^-126 (sum |v| + 1)
to an output: an exponential below 2^-126 may be taken as 0, the largest score's
is 1 or more (no reference lies above it), so after the division an entry's
weight lacks 2^-126 at most; and a result below 2^-126 may be taken as 0 itself.
"""

from __future__ import annotations

import numpy as np
import torch

U16, U32 = 2.0 ** -8, 2.0 ** -24
DROP, LOW, HIGH = 0, 1, 2


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().float().double().numpy() if t.dtype == torch.bfloat16 else t.detach().cpu().double().numpy()


def to_bf16(x: np.ndarray) -> np.ndarray:
    """float64 -> the nearest bf16 (ties to even), as float64: torch's conversion of an exact fp32 value."""
    assert (x == x.astype(np.float32)).all()
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()


def low_values(c: np.ndarray) -> np.ndarray:
    """The values that RETAIN-LOW latents [n, rank] (bf16 values as float64) stand for."""
    x = c.reshape(len(c), -1, 32)
    with np.errstate(over="ignore"):
        s = np.minimum(np.abs(x).max(-1, keepdims=True) / 7.0, 65504.0).astype(np.float16).astype(np.float64)
    q = np.where(s > 0, np.clip(np.rint(x / np.where(s > 0, s, 1.0)), -7, 7), 0.0)
    return to_bf16((q * s).reshape(c.shape))


class Ref:
    """The cache of one layer: per sequence the kept entries in position order, and the counters."""

    def __init__(self, batch, action, floor, n_sink, max_tokens):
        self.act = [max(a, f) for a, f in zip(action, floor)]
        self.n_sink, self.max_tokens = n_sink, max_tokens
        self.rows = [[] for _ in range(batch)]      # (position, store, c, r)
        self.cnt = np.zeros((batch, 6), np.int64)   # n_hi, n_lo, n_pos, n_drop, n_forced, n_lost

    def append(self, b, tags, c, r, keep_all=False):
        """tags: ints or None; c, r: float64 [n, .] of bf16 values."""
        lows = low_values(c) if len(c) else c
        for j in range(len(c)):
            pos = int(self.cnt[b, 2])
            if pos >= self.max_tokens:
                self.cnt[b, 5] += 1
                continue
            tag = 0 if tags is None else int(tags[j])
            forced = keep_all or pos < self.n_sink or tag >= len(self.act)
            a = HIGH if forced else self.act[tag]
            self.cnt[b, 2] += 1
            if a == DROP:
                self.cnt[b, 3] += 1
                continue
            self.cnt[b, 0 if a == HIGH else 1] += 1
            self.cnt[b, 4] += forced
            self.rows[b].append((pos, a, c[j] if a == HIGH else lows[j], r[j]))

    def dense(self, b, rank, rope):
        rows = self.rows[b]
        if not rows:
            return np.zeros((0, rank)), np.zeros((0, rope)), np.zeros(0, np.int64)
        return np.stack([x[2] for x in rows]), np.stack([x[3] for x in rows]), np.array([x[0] for x in rows])


def attention(q, keys, values, scale, seen=None):
    """One head: q [m, d], keys [n, d], values [n, e], seen [m, n] bool or None.  Returns out, lse and the bounds of
    both for a result in bf16 / fp32 (see the module's docstring)."""
    m, n = len(q), len(keys)
    out, lse = np.zeros((m, values.shape[1])), np.full(m, -np.inf)
    out_tol, lse_tol = np.zeros_like(out), np.zeros(m)
    if n == 0:
        return out, lse, out_tol, lse_tol
    s = scale * (q @ keys.T)
    size = abs(scale) * (np.abs(q) @ np.abs(keys).T)
    if seen is None:
        seen = np.ones((m, n), bool)
    s = np.where(seen, s, -np.inf)
    delta = np.where(seen, q.shape[1] * U32 * size + 4 * U32 * np.where(seen, np.abs(s), 0), 0).max(-1)
    some = seen.any(-1)
    top = np.where(some, s.max(-1), 0.0)
    p = np.exp(s - top[:, None])
    total = p.sum(-1)
    p /= np.where(some, total, 1.0)[:, None]
    out = p @ values
    lse = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
    mass = p @ np.abs(values)
    out_tol = 1.05 * (U16 * np.abs(out) + (U16 + 2 * delta + 2.0 ** -22 + n * U32)[:, None] * mass)
    out_tol += 2.0 ** -126 * (seen @ np.abs(values) + 1.0)
    lse_tol = 1.05 * (delta + (n + 16) * U32 + 4 * U32 * np.where(some, np.abs(lse), 0.0))
    return out, lse, out_tol, lse_tol


def check(got, want, tol, what):
    """got within tol of want, where want is finite; equal infinities elsewhere."""
    fin = np.isfinite(want)
    assert (got[~fin] == want[~fin]).all(), f"{what}: infinities differ"
    err = np.abs(got[fin] - want[fin])
    bad = ~(err <= tol[fin] if tol.shape == want.shape else err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} outside the bound, worst {err.max():.3e}"
