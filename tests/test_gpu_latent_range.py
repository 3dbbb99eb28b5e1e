"""Values near the bound that the header gives: an element's magnitudes sum to just less than 2^112 over the entries,
under scores that rise as far as weights can above the reference without moving it."""

import math

import numpy as np
import pytest
import torch

from .latent_ref import HIGH, attention, check, f64
from .test_gpu_latent import DEV, Pair, rnd, run_prompt

pytestmark = pytest.mark.gpu
RISE = 15.9 * math.log(2.0)                          # natural units; the reference moves above 16 log 2


@pytest.mark.parametrize("n, m", [(40, 40), (300, 700)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_prompt(n, m, sign):
    """One score for the first 32 keys, RISE more from there on (bf16 of it: less than 16 log 2)."""
    each = 2.0 ** 112 / (m + 1)

    def edit(q, kv, r):
        q.zero_(), kv[..., :64].zero_(), r.zero_()
        q[..., 0] = 1.0
        kv[32:, :, 0] = RISE
        kv[..., 64:] = sign * each
    assert float(torch.tensor(RISE).bfloat16()) < 16 * math.log(2) and float(torch.tensor(each).bfloat16()) * m < 2.0 ** 112
    o, _ = run_prompt([n], [m], 2, 64, 32, 64, seed=m, spare=0, scale=1.0, edit=edit)
    assert np.isfinite(o).all() and (np.abs(o) > 0.9 * each).all()


@pytest.mark.parametrize("heads", [4, 20, 64, 128])
@pytest.mark.parametrize("n", [300, 4000])
def test_decode(heads, n):
    """The latent's last element is near the bound and the queries leave it out; the rotary keys make the scores."""
    p = Pair(batch=1, heads=heads, rank=128, rope=32, max_tokens=n, seed=n + heads, action=[HIGH], floor=[HIGH],
             scale=1.0)
    tags, c, r = p.tokens(n)
    tags.zero_(), r.zero_()
    c[..., 127] = 2.0 ** 112 / (n + 1)
    assert float(c[0, 0, 127]) * n < 2.0 ** 112
    r[:, 32:, 0] = RISE
    p.append(n, tokens=(tags, c, r))
    q = torch.zeros(1, heads, 160, dtype=torch.bfloat16)
    q[..., 128] = 1.0
    out, _ = p.decode(q)
    assert torch.isfinite(out.float()).all()
