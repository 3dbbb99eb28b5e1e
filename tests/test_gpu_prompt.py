"""Attention of many query tokens over the mixed cache on the GPU, against the
definition in 64 bits within derived bounds (latent_ref, prompt_ref)."""

import math

import numpy as np
import pytest
import torch

from workload.policy import pack_blob, uniform_policy

from . import prompt_ref
from .gpu_util import say
from .latent_ref import check
from .prompt_ref import DROP, HIGH, LOW, f64

pytestmark = pytest.mark.gpu
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
prompt = pytest.importorskip("paper_2608_28276_amd.prompt")
from paper_2608_28276_amd.session import PaskSession  # noqa: E402

SENTINEL = -77.0
N_TAGS = 8


def normal(gen, *shape, gain=1.0):
    return (torch.randn(*shape, generator=gen) * gain).to(torch.bfloat16)


class Run:
    """A session of one layer and the reference beside it."""

    def __init__(self, B, Hq, Hkv, D, max_tokens, actions, n_sink=0, window=0, seed=0, prefill=None, layers=1, layer=0,
                 pages=None):
        pol = uniform_policy(N_TAGS, 1, layers, HIGH)
        for z in range(N_TAGS):
            pol.action[z, 0] = actions[z % len(actions)]
            pol.floor[z, 0] = DROP
        pol.n_sink, pol.recent_window = n_sink, window
        n = B * ((max_tokens + 15) // 16) * layers if pages is None else pages
        self.s = PaskSession(pack_blob(pol), max_batch=B, n_layers=layers, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D,
                             max_tokens_per_seq=max_tokens, hi_pages=n, lo_pages=n, prefill=prefill)
        self.ref = prompt_ref.RefCache(B, [actions[z % len(actions)] for z in range(N_TAGS)], n_sink, window, max_tokens)
        self.B, self.Hq, self.Hkv, self.D, self.layer = B, Hq, Hkv, D, layer
        self.gen = torch.Generator().manual_seed(seed)

    def append(self, n_new, keep_all=False, k=None, v=None):
        m = max(max(n_new), 1)
        k = normal(self.gen, self.B, m, self.Hkv, self.D, gain=1.5) if k is None else k
        v = normal(self.gen, self.B, m, self.Hkv, self.D) if v is None else v
        tags = torch.randint(0, N_TAGS, (self.B, m), generator=self.gen, dtype=torch.uint8)
        self.s.append(self.layer, tags.cuda(), k.cuda(), v.cuda(), n_new=torch.tensor(n_new, dtype=torch.int32).cuda(),
                      keep_all=keep_all)
        for b, n in enumerate(n_new):
            self.ref.append(b, f64(k[b, :n]), f64(v[b, :n]), tags[b, :n], keep_all)

    def attend(self, n_q, first=None, max_q=None, gain=1.0, lse=True, hint=None, scale=None, what=""):
        """One call, checked; returns (out, lse)."""
        m = max_q or max(max(n_q), 1)
        q = normal(self.gen, self.B, m, self.Hq, self.D, gain=gain)
        out = torch.full((self.B, m, self.Hq, self.D), SENTINEL, dtype=torch.bfloat16, device="cuda")
        sums = torch.full((self.B, m, self.Hq), SENTINEL, device="cuda") if lse else None
        if scale is not None:
            self.s.softmax_scale = scale
        say("attend", what, "B", self.B, "Hq", self.Hq, "Hkv", self.Hkv, "D", self.D, "n_q", n_q, "first", first)
        self.s.prompt(self.layer, q.cuda(), out, sums, n_q=torch.tensor(n_q, dtype=torch.int32).cuda(),
                      first=None if first is None else torch.tensor(first, dtype=torch.int32).cuda(), max_ctx_hint=hint)
        torch.cuda.synchronize()
        got, got_lse = f64(out), None if sums is None else f64(sums)
        for b, n in enumerate(n_q):
            n = min(max(n, 0), m)
            at = self.ref.n_pos(b) - n if first is None else first[b]
            want, want_lse, tol, lse_tol = prompt_ref.prompt(self.ref, b, f64(q[b, :n]), at, self.s.softmax_scale)
            check(got[b, :n], want, tol, f"{what} out of sequence {b}")
            assert (got[b, n:] == SENTINEL).all(), f"{what}: rows behind sequence {b} written"
            if lse:
                check(got_lse[b, :n], want_lse, lse_tol, f"{what} lse of sequence {b}")
                assert (got_lse[b, n:] == SENTINEL).all(), f"{what}: lse behind sequence {b} written"
        return out, sums


MIXED = (HIGH, LOW, DROP, LOW, HIGH, LOW, DROP, HIGH)


@pytest.mark.parametrize("Hq, Hkv, D", [(8, 8, 128), (4, 2, 128), (16, 4, 128), (24, 3, 128), (8, 1, 128), (1, 1, 64),
                                        (6, 3, 64), (8, 2, 64), (40, 5, 64)])
@pytest.mark.parametrize("window", [0, 37])
def test_ragged_turns(Hq, Hkv, D, window):
    """Turns of 0 to 300 tokens behind each other, empty sequences among them."""
    r = Run(5, Hq, Hkv, D, 700, MIXED, window=window, n_sink=3, seed=Hq * 100 + D + window)
    for turn in ([1, 0, 17, 300, 64], [2, 0, 63, 1, 65], [130, 1, 16, 15, 31]):
        r.append(turn)
        r.attend(turn, what="turn")
    r.attend([1, 1, 5, 4, 33], lse=False, what="drafts")


@pytest.mark.parametrize("actions", [(HIGH,), (LOW,), (DROP,)])
@pytest.mark.parametrize("window", [0, 16, 200])
def test_single_actions(actions, window):
    r = Run(3, 8, 2, 128, 400, actions, window=window, seed=3)
    r.attend([4, 0, 1], first=[0, 0, 7], what="empty cache")
    r.append([150, 1, 33])
    r.attend([150, 1, 33], what="from the start")
    r.append([90, 0, 1])
    r.attend([90, 2, 1], what="second turn")


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129])
def test_lengths_around_pages_and_steps(n):
    r = Run(2, 4, 1, 128, 300, (HIGH, LOW), seed=n)
    r.append([n, n + 1])
    r.attend([n, n + 1], what="all")
    r.attend([1, 2], what="last")


def test_given_first_positions():
    """Queries before every key, within the history, behind it; far outside of the 32-bit range of positions."""
    r = Run(4, 8, 2, 64, 500, MIXED, window=20, seed=8)
    r.append([400, 400, 100, 0])
    r.attend([70, 70, 70, 3], first=[-60, 120, 90, 0], what="first")
    r.attend([5, 40, 3, 2], first=[-(2 ** 31), 2 ** 31 - 20, 2 ** 31 - 1, 5], what="far")


def test_counts_outside_their_range():
    r = Run(3, 4, 2, 64, 100, MIXED, seed=9)
    r.append([50, 50, 50])
    r.attend([-4, 9, 3], max_q=6, first=[40, 44, 47], what="counts")


@pytest.mark.parametrize("Hq, Hkv", [(8, 1), (8, 8), (16, 4)])
@pytest.mark.parametrize("n_q, hint", [(1, None), (3, None), (8, 256), (40, None), (100, 64)])
def test_long_history_in_pieces(Hq, Hkv, n_q, hint):
    """Few queries over a long mixed history: the keys are cut and joined."""
    r = Run(1, Hq, Hkv, 128, 9000, MIXED, window=50, n_sink=5, seed=n_q)
    r.append([8999 - n_q])
    r.append([n_q])
    r.attend([n_q], hint=hint, what="pieces")
    r.attend([n_q], first=[3000], hint=hint, what="pieces, in the middle")


def test_batch_of_uneven_histories():
    lens = [0, 1, 15, 16, 17, 100, 1023, 2500, 31, 64, 65, 300, 5, 700, 2, 999]
    r = Run(16, 8, 2, 128, 2600, MIXED, seed=12)
    r.append(lens)
    r.attend([min(5, n) for n in lens], max_q=5, what="drafts")
    r.attend([min(70, n) for n in lens], max_q=70, what="turns")


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_scales(scale):
    r = Run(2, 4, 2, 64, 300, MIXED, window=9, seed=13)
    r.append([200, 77])
    r.attend([60, 77], scale=scale, what="scale")


def test_scores_of_hundreds():
    r = Run(1, 4, 2, 128, 900, MIXED, seed=14)
    r.append([800])
    r.attend([300], gain=16.0, what="large scores")
    r.attend([4], gain=16.0, what="large scores")


@pytest.mark.parametrize("prefill", [0x00, 0xFF, 0x7F])
def test_nothing_unwritten_is_read(prefill):
    """Pages, lists and workspaces filled with NaN patterns: partial pages, windows and missing entries show none of it."""
    r = Run(2, 8, 2, 128, 300, MIXED, window=24, seed=15, prefill=prefill)
    r.append([41, 3])
    r.attend([41, 3], what="prefill")
    r.append([100, 10])
    r.attend([7, 2], what="prefill")
    r.append([100, 10])
    r.attend([100, 10], what="prefill")


@pytest.mark.parametrize("n_q", [3, 90])
def test_results_do_not_depend_on_unwritten_bytes(n_q):
    """Bit for bit the same over caches filled with zeros and with NaN patterns."""
    bits = []
    for prefill in (0x00, 0xFF, 0x7F):
        r = Run(2, 8, 2, 128, 300, MIXED, window=21, seed=31, prefill=prefill)
        r.append([150, 97])
        q, out = normal(r.gen, 2, n_q, 8, 128).cuda(), torch.zeros(2, n_q, 8, 128, dtype=torch.bfloat16, device="cuda")
        r.s.prompt(0, q, out)
        bits.append(out.view(torch.int16).cpu())
    assert torch.equal(bits[0], bits[1]) and torch.equal(bits[0], bits[2])


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("n_q", [4, 120])
@pytest.mark.parametrize("window", [0, 40])
def test_hidden_values_that_are_not_finite(value, n_q, window):
    """A kept token's value and key of Inf or NaN reach the queries at its position and behind, no others."""
    r = Run(1, 4, 2, 128, 400, (HIGH,), seed=16, window=window)
    at = 300 - n_q // 2
    k, v = normal(r.gen, 1, 300, 2, 128), normal(r.gen, 1, 300, 2, 128)
    k[0, at, 0, 3], v[0, at, 1, 7] = value, value
    zk, zv = k.clone(), v.clone()
    zk[0, at, 0, 3], zv[0, at, 1, 7] = 0.0, 0.0
    r.s.append(0, None, k.cuda(), v.cuda(), keep_all=True)
    r.ref.append(0, f64(zk[0]), f64(zv[0]), None, True)
    q = normal(r.gen, 1, n_q, 4, 128)
    out = torch.empty(1, n_q, 4, 128, dtype=torch.bfloat16, device="cuda")
    r.s.prompt(0, q.cuda(), out)
    torch.cuda.synchronize()
    m = at - (300 - n_q)                              # queries before the token
    want, _, tol, _ = prompt_ref.prompt(r.ref, 0, f64(q[0, :m]), 300 - n_q, r.s.softmax_scale)
    check(f64(out[0, :m]), want, tol, "before the token")
    assert not np.isfinite(f64(out[0, m:, 2:, 7])).any()      # heads 2 and 3 read KV head 1


@pytest.mark.parametrize("gain", [2.0 ** 11, 2.0 ** 13, 2.0 ** 15])
def test_int4_keys_of_any_size(gain):
    """Keys whose scales 24 of which fp16 does not hold, beside ordinary ones; a key enters as before but for fp16's
    2^-20 in pages with a scale above 2728 (the bound: scale 2^-20 sum |q|, twice for the weights)."""
    r = Run(2, 4, 2, 128, 900, (LOW,), seed=33)
    for n, factor in ((200, 1.0), (64, gain), (130, 1.0), (100, gain)):
        r.append([n, n // 2], k=normal(r.gen, 2, n, 2, 128) * factor)
    r.attend([100, 50], what="keys", scale=2.0 ** -13)
    r.attend([5, 5], what="keys", scale=2.0 ** -13)


@pytest.mark.parametrize("gain", [2.0 ** -12, 2.0 ** 12, 2.0 ** 14, 2.0 ** 17])
def test_int4_values_of_any_size(gain):
    """Values down to fp16's subnormals and beyond its range, in pages of their own and beside ordinary ones."""
    r = Run(2, 4, 2, 128, 900, (LOW,), seed=17)
    for n, factor in ((200, 1.0), (64, gain), (130, 1.0), (100, gain)):
        r.append([n, n // 2], v=normal(r.gen, 2, n, 2, 128) * factor)
    r.attend([100, 50], what="gain")
    r.attend([300, 150], what="gain")
    r.attend([3, 3], what="gain")


def test_int4_scores_are_exact_in_bf16_parts():
    """lse of an int4 history within the bound of fp32 sums, which keys rounded to bf16 miss by far."""
    r = Run(1, 4, 2, 128, 900, (LOW,), seed=32)
    r.append([800])
    _, lse = r.attend([100], what="exact scores")
    want = prompt_ref.prompt(r.ref, 0, np.zeros((1, 4, 128)), 799, 1.0)[1]
    assert np.allclose(want, math.log(800)) and lse.shape == (1, 100, 4)


def test_one_query_agrees_with_the_decode_call():
    r = Run(6, 16, 4, 128, 600, MIXED, window=30, seed=18)
    r.append([1, 50, 100, 299, 400, 600])
    q = normal(r.gen, 6, 1, 16, 128).cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    la, lb = torch.empty(6, 1, 16, device="cuda"), torch.empty(6, 1, 16, device="cuda")
    r.s.prompt(0, q, a, la)
    r.s.decode(0, q.view(6, 16, 128), b.view(6, 16, 128), lb.view(6, 16))
    torch.cuda.synchronize()
    assert (f64(a) - f64(b) <= 2e-3 + 1e-2 * np.abs(f64(b))).all() and np.abs(f64(la) - f64(lb)).max() < 2e-2


def test_layers_and_sequences_do_not_mix():
    r = Run(3, 8, 2, 64, 200, MIXED, seed=19, layers=3, layer=1)
    other = Run(3, 8, 2, 64, 200, MIXED, seed=20, layers=3, layer=2)
    other.s = r.s
    r.append([100, 7, 64])
    other.append([3, 150, 0])
    r.attend([50, 7, 64], what="layer 1")
    other.attend([3, 90, 0], what="layer 2")


def test_the_cache_is_not_modified_and_calls_repeat():
    r = Run(3, 16, 2, 128, 900, MIXED, window=33, seed=21)
    r.append([800, 1, 300])
    before = r.s.buf.clone()
    for n_q in ([5, 1, 3], [300, 1, 300]):
        m = max(n_q)
        q = normal(r.gen, 3, m, 16, 128).cuda()
        outs = []
        for _ in range(2):
            out, lse = torch.zeros_like(q), torch.zeros(3, m, 16, device="cuda")
            r.s.prompt(0, q, out, lse, n_q=torch.tensor(n_q, dtype=torch.int32).cuda())
            outs.append((out, lse))
        assert torch.equal(outs[0][0].view(torch.int16), outs[1][0].view(torch.int16))
        assert torch.equal(outs[0][1].view(torch.int32), outs[1][1].view(torch.int32))
    assert torch.equal(before, r.s.buf)


def test_graph_replays_of_a_whole_turn():
    """Rotate at the cache's own positions, append, attend, captured once for two layers: every replay is the next turn
    and equals the eager calls on a second session."""
    rope = prompt.make_rope(128, 1e6)
    B, m, Hq, Hkv, D = 2, 6, 8, 2, 128
    runs = [Run(B, Hq, Hkv, D, 900, MIXED, window=10, seed=22, layers=2) for _ in range(2)]
    gen = torch.Generator().manual_seed(23)
    for layer in range(2):
        k, v = normal(gen, B, 300, Hkv, D).cuda(), normal(gen, B, 300, Hkv, D).cuda()
        tags = torch.randint(0, N_TAGS, (B, 300), generator=gen, dtype=torch.uint8).cuda()
        for r in runs:
            r.s.append(layer, tags, k, v)
    rows = torch.zeros(B, m, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device="cuda")
    tags = torch.zeros(B, m, dtype=torch.uint8, device="cuda")
    n_new = torch.full((B,), m, dtype=torch.int32, device="cuda")
    made = lambda h: torch.zeros(B, m, h, D, dtype=torch.bfloat16, device="cuda")

    def turn(s, bufs):
        q_in = rows[:, :, :Hq * D].unflatten(2, (Hq, D))
        k_in = rows[:, :, Hq * D:(Hq + Hkv) * D].unflatten(2, (Hkv, D))
        v = rows[:, :, (Hq + Hkv) * D:].unflatten(2, (Hkv, D)).contiguous()
        for layer, (q, k, out, lse) in enumerate(bufs):
            s.rotate(rope, layer, q_in, q, k_in, k, n_new=n_new)
            s.append(layer, tags, k, v, n_new=n_new)
            s.prompt(layer, q, out, lse, n_q=n_new)

    bufs = [[(made(Hq), made(Hkv), made(Hq), torch.zeros(B, m, Hq, device="cuda")) for _ in range(2)] for _ in runs]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        turn(runs[0].s, bufs[0])
    for step in range(4):
        rows.copy_(normal(gen, *rows.shape))
        tags.copy_(torch.randint(0, N_TAGS, tags.shape, generator=gen, dtype=torch.uint8))
        n_new.copy_(torch.tensor([m, step + 1], dtype=torch.int32))
        graph.replay()
        turn(runs[1].s, bufs[1])
        torch.cuda.synchronize()
        for layer, (x, y) in enumerate(zip(bufs[0], bufs[1])):
            for name, t, u in zip(("q", "k", "out", "lse"), x, y):
                assert torch.equal(t, u), f"step {step}, layer {layer}, {name}: {int((t != u).sum())} differ"
    assert torch.equal(runs[0].s.next_positions(0), runs[1].s.next_positions(1))
    assert runs[0].s.next_positions(0).tolist() == [300 + 4 * m, 300 + 1 + 2 + 3 + 4]


def test_a_turn_from_projections_against_the_definition():
    """Rotate, append, attend, each checked by what the definition makes of the call before it."""
    B, Hq, Hkv, D = 2, 8, 2, 64
    r = Run(B, Hq, Hkv, D, 400, MIXED, seed=24, window=12)
    rope, freq = prompt.make_rope(D, 1e4), prompt_ref.frequencies(D, 1e4)
    for turn in ([150, 20], [40, 1], [0, 33]):
        m = max(turn)
        q, k, v = (normal(r.gen, B, m, h, D) for h in (Hq, Hkv, Hkv))
        n_new = torch.tensor(turn, dtype=torch.int32).cuda()
        q_rot, k_rot = torch.zeros_like(q).cuda(), torch.zeros_like(k).cuda()
        starts = r.s.next_positions(0).cpu().numpy()
        r.s.rotate(rope, 0, q.cuda(), q_rot, k.cuda(), k_rot, n_new=n_new)
        torch.cuda.synchronize()
        for b, n in enumerate(turn):
            for got, x in ((q_rot, q), (k_rot, k)):
                want, tol = prompt_ref.rotate(f64(x[b, :n]), starts[b] + np.arange(n), freq, 0, D, False)
                assert (np.abs(f64(got[b, :n]) - want) <= tol).all()
        tags = torch.randint(0, N_TAGS, (B, m), generator=r.gen, dtype=torch.uint8)
        r.s.append(0, tags.cuda(), k_rot, v.cuda(), n_new=n_new)
        for b, n in enumerate(turn):
            r.ref.append(b, f64(k_rot[b, :n]), f64(v[b, :n]), tags[b, :n])
        out, lse = torch.full_like(q_rot, SENTINEL), torch.zeros(B, m, Hq, device="cuda")
        r.s.prompt(0, q_rot, out, lse, n_q=n_new)
        torch.cuda.synchronize()
        for b, n in enumerate(turn):
            want, want_lse, tol, lse_tol = prompt_ref.prompt(r.ref, b, f64(q_rot[b, :n]), r.ref.n_pos(b) - n,
                                                             r.s.softmax_scale)
            check(f64(out[b, :n]), want, tol, "turn")
            check(f64(lse[b, :n]), want_lse, lse_tol, "turn's lse")


def test_full_pools_and_full_sequences():
    """Tokens that found no page, or no position, are not there to attend; the rest is."""
    r = Run(1, 4, 2, 64, 100, (HIGH,), seed=25, pages=4)
    k, v = normal(r.gen, 1, 90, 2, 64), normal(r.gen, 1, 90, 2, 64)
    r.s.append(0, None, k.cuda(), v.cuda(), keep_all=True)      # 4 pages hold 64 of the 90
    r.ref.append(0, f64(k[0, :64]), f64(v[0, :64]), None, True)
    r.attend([50], first=[40], what="full pool")
    r = Run(1, 4, 2, 64, 70, (HIGH, LOW), seed=26)
    k, v = normal(r.gen, 1, 60, 2, 64), normal(r.gen, 1, 60, 2, 64)
    r.append([60], k=k, v=v)
    r.append([20])                                    # 10 of them find a position
    r.attend([20], first=[60], what="full sequence")


def test_another_stream_and_two_sessions():
    a, b = Run(2, 8, 2, 128, 500, MIXED, seed=27), Run(2, 4, 4, 64, 500, MIXED, seed=28)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.append([400, 90])
        b.append([80, 333])
        a.attend([4, 4], what="a")
        b.attend([70, 200], what="b")
    s.synchronize()


def test_many_tiles():
    """More rows than a tile holds in every sequence, with a wave that starts past the last row."""
    r = Run(2, 8, 1, 64, 700, MIXED, seed=29, window=5)
    r.append([650, 33])
    r.attend([650, 33], what="tiles")


def test_refusals_of_tensors():
    r = Run(2, 8, 2, 128, 100, MIXED, seed=30)
    q, out = torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16,
                                                                                       device="cuda")
    n = torch.ones(2, dtype=torch.int32, device="cuda")

    def status(*args, **kw):
        with pytest.raises(pask.PaskError) as e:
            r.s.prompt(*args, **kw)
        return e.value.status

    ARG, SHAPE = pask.PASK_E_ARG, pask.PASK_E_SHAPE
    assert status(0, q.float(), out) == ARG
    assert status(0, q.cpu(), out) == ARG
    assert status(0, q, out[:, :2]) == ARG            # strided
    assert status(0, q, out[:1]) == SHAPE
    assert status(0, q[:, :, :4].contiguous(), out) == SHAPE
    assert status(0, q, out, torch.zeros(2, 3, 4, device="cuda")) == SHAPE
    assert status(0, q, out, n_q=n.long()) == ARG
    assert status(0, q, out, n_q=n[:1]) == SHAPE
    assert status(0, q, out, first=n.float()) == ARG
    assert status(1, q, out) == SHAPE
    big = torch.zeros(3, 3, 8, 128, dtype=torch.bfloat16, device="cuda")
    assert status(0, big, big) == SHAPE
    long = torch.zeros(1, 101, 8, 128, dtype=torch.bfloat16, device="cuda")
    assert status(0, long, long) == SHAPE
    r.s.prompt(0, q[:, :0].contiguous(), out[:, :0].contiguous())
