"""Calls of up to 32 rows (query tokens times query heads of a KV head), a
draft's: the weights of HIGH values count with 16 bits, as those of the decode
call do.

Bounds: latent_ref's, in which a weight's rounding to bf16, u16 = 2^-8 of it, is
replaced by that of two bf16 parts: the first leaves 2^-8 of the weight at most,
exactly (a difference of nearby fp32 numbers), and the second's rounding 2^-8 of
that, 2^-16.  The outputs' own rounding, u16 |o|, stays."""

import numpy as np
import pytest
import torch

from . import latent_ref, prompt_ref
from .gpu_util import say
from .latent_ref import U16, check
from .prompt_ref import HIGH, f64

pytestmark = pytest.mark.gpu
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
from .test_gpu_prompt import MIXED, Run, normal  # noqa: E402


def fine(q, k, v, scale, seen):
    want, lse, tol, lse_tol = latent_ref.attention(q, k, v, scale, seen)
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    mass = np.where(np.isfinite(lse)[:, None], np.exp(s - np.where(np.isfinite(lse), lse, 0.0)[:, None]), 0.0) @ np.abs(v)
    return want, lse, tol - 1.05 * (U16 - 2.0 ** -16) * mass, lse_tol


@pytest.mark.parametrize("Hq, Hkv, n_q", [(8, 8, 32), (4, 2, 16), (8, 2, 5), (8, 1, 4), (8, 1, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window, n", [(0, 37), (0, 700), (50, 700), (0, 3000)])
def test_drafts_weights_count_with_16_bits(Hq, Hkv, n_q, D, window, n):
    r = Run(1, Hq, Hkv, D, 3100, (HIGH,), seed=Hq + n_q + D + n, window=window)
    r.append([n])
    q = normal(r.gen, 1, n_q, Hq, D)
    out = torch.full((1, n_q, Hq, D), -77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((1, n_q, Hq), -77.0, device="cuda")
    say("draft", Hq, Hkv, n_q, D, window, n)
    r.s.prompt(0, q.cuda(), out, lse)
    torch.cuda.synchronize()
    pos, k, v = r.ref.visible(0)
    seen = pos[None] <= n - n_q + np.arange(n_q)[:, None]
    for h in range(Hq):
        g = h * Hkv // Hq
        want, want_lse, tol, lse_tol = fine(f64(q[0, :, h]), k[:, g], v[:, g], r.s.softmax_scale, seen)
        check(f64(out[0, :, h]), want, tol, f"out of head {h}")
        check(f64(lse[0, :, h]), want_lse, lse_tol, f"lse of head {h}")


def test_one_query_and_the_decode_call_are_both_within_the_bounds():
    """Also each other, on both sides: no further apart than their bounds together."""
    r = Run(6, 16, 4, 128, 600, MIXED, window=30, seed=18)
    r.append([1, 50, 100, 299, 400, 600])
    q = normal(r.gen, 6, 1, 16, 128)
    a, b = (torch.empty(6, 1, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    la, lb = torch.empty(6, 1, 16, device="cuda"), torch.empty(6, 1, 16, device="cuda")
    r.s.prompt(0, q.cuda(), a, la)
    r.s.decode(0, q.cuda().view(6, 16, 128), b.view(6, 16, 128), lb.view(6, 16))
    torch.cuda.synchronize()
    for i in range(6):
        want, want_lse, tol, lse_tol = prompt_ref.prompt(r.ref, i, f64(q[i]), r.ref.n_pos(i) - 1, r.s.softmax_scale)
        for name, out, lse in (("prompt", a, la), ("decode", b, lb)):
            check(f64(out[i]), want, tol, f"{name}: out of sequence {i}")
            check(f64(lse[i]), want_lse, lse_tol, f"{name}: lse of sequence {i}")
        assert (np.abs(f64(a[i]) - f64(b[i])) <= 2 * tol).all() and (np.abs(f64(la[i]) - f64(lb[i])) <= 2 * lse_tol).all()
