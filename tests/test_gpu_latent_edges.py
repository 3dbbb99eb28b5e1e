"""Latent operators where they could go wrong in ways of their own: references that move at every head count, values
near the largest, entries lost to full pools, batches past the ranking of prompt tiles."""
import math

import numpy as np
import pytest
import torch

from .latent_ref import HIGH, LOW, attention, check, f64
from .test_gpu_latent import DEV, Pair, latent, pask, rnd, run_prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [128, 512])
@pytest.mark.parametrize("heads", [1, 16, 30, 64, 128])
def test_decode_of_rising_scores(rank, heads):
    """The reference moves again and again, in every layout of heads over waves."""
    p = Pair(batch=2, heads=heads, rank=rank, max_tokens=500, seed=heads + rank)
    tags, c, r = p.tokens(400)
    ramp = torch.linspace(0.01, 6.0, 400)[None, :, None]
    p.append(400, tokens=(tags, (c.float() * ramp).to(torch.bfloat16), r))
    p.decode(p.queries(scale=4.0))


@pytest.mark.parametrize("nq, nk", [([40], [40]), ([300], [700])])
def test_prompt_of_huge_values(nq, nk):
    """Values up to 1e30, which weights far above 1 would carry past the largest fp32; scores rise along the keys."""
    def edit(q, kv, r):
        kv[..., 64:] = (kv[..., 64:].float() * 1e29).to(torch.bfloat16)
        q[..., :64] = 1.0
        kv[..., :64] = torch.linspace(0.0, 1.5, len(kv))[:, None, None].to(torch.bfloat16)
    o, _ = run_prompt(nq, nk, 2, 64, 32, 64, seed=9, spare=0, scale=1.0, edit=edit)
    assert np.isfinite(o).all() and np.abs(o).max() > 1e28


def test_read_and_decode_after_losses():
    """A full pool loses its store's tokens and no others; what is kept reads back in order and is attended."""
    p = Pair(batch=1, rank=128, rope=32, max_tokens=300, hi_pages=2, lo_pages=3, seed=5)
    p.append(200)
    p.append(1)
    hi, lo = [x for x in p.ref.rows[0] if x[1] == HIGH], [x for x in p.ref.rows[0] if x[1] == LOW]
    assert len(hi) > 32 and len(lo) > 48
    kept = sorted(hi[:32] + lo[:48], key=lambda x: x[0])
    c = torch.full((90, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    r = torch.full((90, 32), 7.0, dtype=torch.bfloat16, device=DEV)
    pos, cu = torch.zeros(90, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    p.sess.read(0, c, r, pos, cu)
    assert cu.cpu().tolist() == [0, 80]
    assert pos[:80].cpu().tolist() == [x[0] for x in kept]
    assert (f64(c)[:80] == np.stack([x[2] for x in kept])).all() and (f64(r)[:80] == np.stack([x[3] for x in kept])).all()
    assert (c[80:] == 7.0).all() and (r[80:] == 7.0).all()
    q = p.queries()
    out, lse = torch.empty(1, 16, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 16, device=DEV)
    p.sess.decode(0, q.to(DEV), out, lse)
    keys = np.concatenate([f64(c)[:80], f64(r)[:80]], 1)
    o, l, to, tl = attention(f64(q)[0], keys, f64(c)[:80], p.scale)
    check(f64(out)[0], o, to, "out")
    check(f64(lse)[0], l, tl, "lse")


@pytest.mark.parametrize("batch, most", [(63, 60), (64, 60), (65, 60), (130, 9), (12, 700), (40, 300)])
def test_prompt_batches(batch, most):
    """As many tiles as are ranked by their length, and more; every sequence of another length, some empty."""
    g = np.random.default_rng(batch)
    nq = [int(x) for x in g.integers(0, most + 1, batch)]
    nq[3] = most
    nk = [int(n + x) for n, x in zip(nq, g.integers(0, 90, batch))]
    run_prompt(nq, nk, 1, 64, 32, 64, seed=batch)


def test_prompt_in_chunks_is_the_whole_prompt():
    """Chunks of a prompt, each after the ones before it, against the prompt at once (other tiles, other order)."""
    g = torch.Generator().manual_seed(3)
    n, heads = 700, 3
    q, kv, r = rnd(g, n, heads, 192).to(DEV), rnd(g, n, heads, 256).to(DEV), rnd(g, n, 64).to(DEV)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    whole, parts = (torch.empty(n, heads, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    latent.prompt_attn(q, kv, r, whole, None, cu, cu, n)
    at = 0
    for m in (1, 40, 300, 359):
        cq, ck = (torch.tensor([0, x], dtype=torch.int32, device=DEV) for x in (m, at + m))
        latent.prompt_attn(q[at:at + m], kv[:at + m], r[:at + m], parts[at:at + m], None, cq, ck, m)
        at += m
    f = lambda x: f64(x)
    for h in range(heads):
        keys = np.concatenate([f(kv)[:, h, :128], f(r)], 1)
        seen = np.arange(n)[None] <= np.arange(n)[:, None]
        want = attention(f(q)[:, h], keys, f(kv)[:, h, 128:], 1.0 / math.sqrt(192), seen)
        check(f(whole)[:, h], want[0], want[2], f"whole, head {h}")
        check(f(parts)[:, h], want[0], want[2], f"parts, head {h}")


def test_refusals_of_a_token_without_tags_and_of_scales():
    p = Pair(batch=2, rank=128, rope=32, heads=4)
    q, out = p.queries().to(DEV), torch.empty(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    _, c, r = (x.to(DEV) for x in p.tokens(1))
    with pytest.raises(pask.PaskError):
        p.sess.decode(0, q, out, c_new=c[:, 0].contiguous(), r_new=r[:, 0].contiguous())
    for scale in (3e38, -3e38, math.inf, math.nan):
        p.sess.softmax_scale = scale
        with pytest.raises(pask.PaskError):
            p.sess.decode(0, q, out)
    p.check_counters()
