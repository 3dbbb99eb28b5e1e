"""Prompts over keys at given positions against the plain 64-bit reference, and the turn of a chat whose table drops
tokens: what a query sees is what was kept at its position and before."""

import math

import numpy as np
import pytest
import torch

from .latent_ref import DROP, HIGH, LOW, attention, check, f64
from .test_gpu_latent import DEV, PROMPT_DIMS, Pair, latent, pask, rnd

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Prompts:
    """Sequences of nq[b] queries from position first[b] on, and keys at positions pos[b]."""

    def __init__(self, nq, first, pos, heads=2, nope=64, rope=32, v=64, seed=0, spare=2, edit=None):
        g = torch.Generator().manual_seed(seed)
        self.nq, self.first, self.pos = nq, first, [np.asarray(p, np.int64) for p in pos]
        self.heads, self.nope, self.v, self.scale = heads, nope, v, 1.0 / math.sqrt(nope + rope)
        self.cq, self.ck = np.cumsum([0] + list(nq)), np.cumsum([0] + [len(p) for p in pos])
        tq, tk = int(self.cq[-1]) + spare, int(self.ck[-1]) + spare
        self.q, self.kv, self.r = rnd(g, tq, heads, nope + rope), rnd(g, tk, heads, nope + v), rnd(g, tk, rope)
        self.kv[int(self.ck[-1]):], self.r[int(self.ck[-1]):] = float("nan"), float("nan")
        if edit:
            edit(self)
        self.dev = [x.to(DEV) for x in (self.q, self.kv, self.r)]
        self.cu = [i32(self.cq), i32(self.ck)]
        self.at = dict(pos=i32(np.concatenate(self.pos + [np.zeros(spare)])), q_first=i32(first))

    def outputs(self):
        tq = len(self.q)
        return (torch.full((tq, self.heads, self.v), 7.0, dtype=torch.bfloat16, device=DEV),
                torch.full((tq, self.heads), 7.0, device=DEV))

    def run(self, max_q=None):
        out, lse = self.outputs()
        latent.prompt_attn(*self.dev, out, lse, *self.cu, max(self.nq) if max_q is None else max_q, **self.at)
        return out, lse

    def check(self, out, lse, max_q=None):
        q, kv, r, o, l = f64(self.q), f64(self.kv), f64(self.r), f64(out), f64(lse)
        for b, n in enumerate(self.nq):
            done = n if max_q is None else min(n, max_q)
            a, z = self.cq[b], self.cq[b] + done
            k = slice(self.ck[b], self.ck[b + 1])
            seen = self.pos[b][None] <= self.first[b] + np.arange(done)[:, None]
            for h in range(self.heads):
                keys = np.concatenate([kv[k, h, :self.nope], r[k]], 1)
                want = attention(q[a:z, h], keys, kv[k, h, self.nope:], self.scale, seen)
                check(o[a:z, h], want[0], want[2], f"out of sequence {b}, head {h}")
                check(l[a:z, h], want[1], want[3], f"lse of sequence {b}, head {h}")
            blind = ~seen.any(1)
            assert (o[a:z][blind] == 0).all() and (l[a:z][blind] == -math.inf).all()
            assert (o[z:self.cq[b + 1]] == 7.0).all()
        assert (o[self.cq[-1]:] == 7.0).all() and (l[self.cq[-1]:] == 7.0).all()


def kept(g, n, share):
    """Positions of n tokens of which about this share is kept."""
    return np.flatnonzero(g.random(n) < share)


@pytest.mark.parametrize("nope, rope, v", PROMPT_DIMS)
def test_every_size(nope, rope, v):
    g = np.random.default_rng(nope + rope + v)
    nq, past = [1, 64, 0, 65, 130, 33], [0, 7, 20, 300, 63, 64]
    p = Prompts(nq, past, [kept(g, m + n, 0.6) for n, m in zip(nq, past)], 3, nope, rope, v, seed=1)
    p.check(*p.run())


@pytest.mark.parametrize("n, past", [(1, 0), (1, 999), (40, 0), (64, 700), (65, 30), (256, 0), (257, 2000), (700, 1500)])
@pytest.mark.parametrize("share", [0.0, 0.1, 0.5, 0.9])
def test_lengths(n, past, share):
    g = np.random.default_rng(n + past)
    p = Prompts([n], [past], [kept(g, past + n, share)], seed=n)
    p.check(*p.run())


@pytest.mark.parametrize("n", [30, 300])
@pytest.mark.parametrize("what", ["turn dropped", "history dropped", "tail dropped", "head dropped", "one kept"])
def test_runs_of_drops(n, what):
    past = 97
    k = {"turn dropped": np.arange(past), "history dropped": past + np.arange(n), "tail dropped": np.arange(past + n // 2),
         "head dropped": np.arange(past // 2, past + n), "one kept": np.array([past + n // 2])}[what]
    p = Prompts([n], [past], [k], seed=n)
    p.check(*p.run())


@pytest.mark.parametrize("n, past", [(50, 0), (50, 77), (400, 0), (300, 1111)])
def test_nothing_dropped_is_the_place_from_the_end(n, past):
    """With every token kept the keys' positions and their places say the same: equal bit for bit."""
    p = Prompts([n, 20], [past, 5], [np.arange(past + n), np.arange(25)], 3, 128, 64, 128, seed=past)
    out, lse = p.run()
    p.check(out, lse)
    want, want_l = p.outputs()
    latent.prompt_attn(*p.dev, want, want_l, *p.cu, max(p.nq))
    assert torch.equal(out, want) and torch.equal(lse, want_l)


def test_positions_at_their_ends():
    """The largest positions, queries before every key and behind the largest position, positions that repeat."""
    top = 2 ** 31 - 1
    pos = [np.arange(top - 39, top + 1), np.arange(100, 140), np.repeat(np.arange(20), 2), np.arange(40)]
    p = Prompts([40, 40, 40, 40], [top - 39, 70, 0, -20], pos, seed=5)
    p.check(*p.run())
    p = Prompts([40, 40], [top - 5, -2 ** 31], pos[:2], seed=6)
    p.check(*p.run())


def test_computes_max_q_queries():
    g = np.random.default_rng(3)
    p = Prompts([300, 20, 150], [10, 0, 90], [kept(g, m, 0.5) for m in (310, 20, 240)], seed=3)
    p.check(*p.run(max_q=130), max_q=130)


@pytest.mark.parametrize("batch, most", [(64, 60), (65, 60), (130, 9), (12, 700)])
def test_batches(batch, most):
    g = np.random.default_rng(batch)
    nq = [int(x) for x in g.integers(0, most + 1, batch)]
    nq[3] = most
    past = [int(x) for x in g.integers(0, 200, batch)]
    p = Prompts(nq, past, [kept(g, n + m, g.random()) for n, m in zip(nq, past)], 1, seed=batch)
    p.check(*p.run())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.3895313892515355e38])
def test_bad_keys_behind_a_query(bad):
    """A bad key or value leaves every query at an earlier position as it is."""
    pos = np.sort(np.random.default_rng(7).permutation(240)[:150])
    at = 90                                          # queries at positions below pos[at] do not see it
    blind = int(pos[at]) - 40

    def spoil(p):
        p.kv[at], p.r[at] = bad, bad
    p = Prompts([200], [40], [pos], 4, 128, 64, 128, seed=8, edit=spoil)
    out, lse = p.run()
    clean = Prompts([200], [40], [pos], 4, 128, 64, 128, seed=8)
    p.kv, p.r, p.nq = clean.kv, clean.r, [blind]
    p.cq = np.array([0, blind])
    p.check(torch.cat([out[:blind], out[200:]]), torch.cat([lse[:blind], lse[200:]]))


def test_offsets_outside_the_rows_and_unsorted_positions():
    """Nothing outside the rows is read or written; another sequence's disorder changes nothing."""
    q, kv, r = (torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((20, 2, 96), (20, 2, 128), (20, 32)))
    out = torch.full((20, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    cu = i32([-4, 9, 5, 90])
    latent.prompt_attn(q, kv, r, out, None, cu, cu, 20, pos=i32(np.arange(20)), q_first=i32([0, 5, 5]))
    assert (out == 0).all()
    g = np.random.default_rng(1)
    p = Prompts([100, 100], [60, 60], [g.permutation(160), np.arange(0, 160, 2)], seed=2)
    out, lse = p.run()
    assert torch.isfinite(out.float()).all()
    p.q, p.kv, p.r = p.q[100:], p.kv[160:], p.r[160:]
    p.nq, p.first, p.pos = [100], [60], p.pos[1:]
    p.cq, p.ck = np.array([0, 100]), np.array([0, 80])
    p.check(out[100:], lse[100:])


def test_refusals():
    p = Prompts([5], [3], [np.arange(6)])
    out, lse = p.outputs()
    pos, first = p.at["pos"], p.at["q_first"]
    for at in (dict(pos=pos), dict(q_first=first), dict(pos=pos.long(), q_first=first), dict(pos=pos[:-1], q_first=first),
               dict(pos=pos, q_first=first.repeat(2)), dict(pos=pos.cpu(), q_first=first),
               dict(pos=pos.repeat(2)[::2], q_first=first)):
        with pytest.raises(pask.PaskError):
            latent.prompt_attn(*p.dev, out, lse, *p.cu, 5, **at)
    assert (out == 7.0).all()
    s = Pair(batch=2, rank=128, rope=32, heads=4).sess
    for bad in (dict(layer=1), dict(layer=-1), dict(layer=0, batch=3), dict(layer=0, batch=0)):
        with pytest.raises(pask.PaskError):
            s.next_positions(**bad)


def turn(p, lens, heads, w_kv, v, q, keep_all=False):
    """One turn of a chat: the tokens persisted, all kept ones read back, expanded and attended.  Returns out, lse."""
    nope = w_kv.shape[1] - v
    first = p.sess.next_positions(p.layer)
    assert first.tolist() == p.ref.cnt[:, 2].tolist()
    p.append(lens, keep_all=keep_all)
    rows = int(p.ref.cnt[:, :2].sum()) + 5           # room behind the last row
    c = torch.full((rows, p.rank), float("nan"), dtype=torch.bfloat16, device=DEV)
    r = torch.full((rows, p.rope), float("nan"), dtype=torch.bfloat16, device=DEV)
    pos, cu_k = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.empty(p.batch + 1, dtype=torch.int32, device=DEV)
    p.sess.read(p.layer, c, r, pos, cu_k)
    kv = torch.from_numpy(np.einsum("tr,hnr->thn", f64(c), w_kv)).to(torch.bfloat16).to(DEV)
    cq = np.cumsum([0] + list(lens))
    out, lse = torch.empty(cq[-1], heads, v, dtype=torch.bfloat16, device=DEV), torch.empty(cq[-1], heads, device=DEV)
    p.sess.prompt(q.to(DEV), kv, r, out, lse, i32(cq), cu_k, max(lens), pos=pos, q_first=first)
    kv, q, o, l = f64(kv), f64(q), f64(out), f64(lse)
    at = 0
    for b, n in enumerate(lens):
        _, rope, where = p.ref.dense(b, p.rank, p.rope)       # kept entries of every turn so far, in position order
        seen = where[None] <= int(first[b]) + np.arange(n)[:, None]
        k = slice(at, at + len(where))
        for h in range(heads):
            keys = np.concatenate([kv[k, h, :nope], rope], 1)
            want = attention(q[cq[b]:cq[b + 1], h], keys, kv[k, h, nope:], p.scale, seen)
            check(o[cq[b]:cq[b + 1], h], want[0], want[2], f"out of sequence {b}, head {h}")
            check(l[cq[b]:cq[b + 1], h], want[1], want[3], f"lse of sequence {b}, head {h}")
        at += len(where)
    return out, lse


@pytest.mark.parametrize("action", [[HIGH, LOW, DROP, LOW, DROP], [HIGH, DROP], [LOW, DROP, DROP], [DROP]])
def test_turns_whose_table_drops_tokens(action):
    """Turns of several sequences by the table, the last of one token, which a decode step at its position agrees with."""
    heads, nope, rank, rope, v = 6, 64, 256, 32, 64
    p = Pair(batch=3, heads=heads, rank=rank, rope=rope, max_tokens=700, seed=21, scale=1 / math.sqrt(nope + rope),
             action=action, floor=[DROP] * len(action), n_sink=2)
    g = torch.Generator().manual_seed(22)
    w_kv = (torch.randn(heads, nope + v, rank, generator=g) / 16).double().numpy()
    for lens in ([70, 33, 1], [64, 0, 300], [5, 257, 40], [1, 1, 1]):
        q = rnd(g, sum(lens), heads, nope + rope)
        out, _ = turn(p, lens, heads, w_kv, v, q)
    q_abs = torch.from_numpy(np.concatenate([np.einsum("bhn,hnr->bhr", f64(q)[:, :, :nope], w_kv[:, :nope]),
                                             f64(q)[:, :, nope:]], 2)).to(torch.bfloat16)
    absorbed, _ = p.decode(q_abs)                    # over the same entries: the last token is in the cache
    got = np.einsum("bhr,hvr->bhv", f64(absorbed), w_kv[:, nope:])
    for b in range(3):
        c, r, _ = p.ref.dense(b, rank, rope)
        for h in range(heads):
            # the absorbed query and the expanded keys and values were rounded to bf16: scores move by at most
            # 2^-8 (sum |q_abs c| + sum |q k|), so weights by a factor within e^(2 delta); each of the two results has
            # three more roundings to bf16 of at most 2^-8 of sum |w c| (its weights, values and output)
            k = np.concatenate([c @ w_kv[h, :nope].T, r], 1)
            delta = p.scale * 2 ** -8 * ((np.abs(f64(q_abs)[b, h]) @ np.abs(np.concatenate([c, r], 1)).T).max() +
                                         (np.abs(f64(q)[b, h]) @ np.abs(k).T).max())
            mass = np.abs(w_kv[h, nope:]) @ np.abs(c).max(0)
            assert (np.abs(got[b, h] - f64(out)[b, h]) <= (2 * delta * math.exp(2 * delta) + 6 * 2 ** -8) * mass).all()


def test_a_turn_in_a_graph():
    """Persist, read back and attend captured once; replayed on other tokens with eager work between."""
    heads, n = 4, 40
    p = Pair(batch=2, heads=heads, rank=128, rope=32, max_tokens=600, seed=31)
    p.append([30, 90])
    g = torch.Generator().manual_seed(32)
    rows = 600
    c, r = (torch.zeros(rows, x, dtype=torch.bfloat16, device=DEV) for x in (128, 32))
    pos, cu_k = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    kv, q = rnd(g, rows, heads, 128).to(DEV), rnd(g, 2 * n, heads, 96).to(DEV)     # some expansion, the same each time
    out, lse = torch.empty(2 * n, heads, 64, dtype=torch.bfloat16, device=DEV), torch.empty(2 * n, heads, device=DEV)
    cu_q = i32([0, n, 2 * n])
    tags, tc, tr = (x.to(DEV) for x in p.tokens(n))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = p.sess.next_positions(0)
        p.sess.append(0, tags, tc, tr)
        p.sess.read(0, c, r, pos, cu_k)
        p.sess.prompt(q, kv, r, out, lse, cu_q, cu_k, n, pos=pos, q_first=first)
    for _ in range(4):
        new = p.tokens(n)
        tags.copy_(new[0]), tc.copy_(new[1]), tr.copy_(new[2])
        start = p.ref.cnt[:, 2].copy()
        for b in range(2):
            p.ref.append(b, new[0][b].numpy(), f64(new[1][b]), f64(new[2][b]))
        graph.replay()
        torch.cuda.synchronize()
        assert first.tolist() == start.tolist()
        want, want_l = torch.empty_like(out), torch.empty_like(lse)
        p.sess.prompt(q, kv, r, want, want_l, cu_q, cu_k, n, pos=pos, q_first=i32(start))
        assert torch.equal(out, want) and torch.equal(lse, want_l)
        ck = cu_k.tolist()
        assert pos[:ck[2]].tolist() == [int(x) for b in range(2) for x in p.ref.dense(b, 128, 32)[2]]
        for b in range(2):
            where = p.ref.dense(b, 128, 32)[2]
            seen = where[None] <= start[b] + np.arange(n)[:, None]
            for h in range(heads):
                k = slice(ck[b], ck[b + 1])
                keys = np.concatenate([f64(kv)[k, h, :64], f64(r)[k]], 1)
                w = attention(f64(q)[b * n:b * n + n, h], keys, f64(kv)[k, h, 64:], p.scale, seen)
                check(f64(out)[b * n:b * n + n, h], w[0], w[2], "out")
        p.append([3, 5])                             # eager work between
    p.check_counters()
