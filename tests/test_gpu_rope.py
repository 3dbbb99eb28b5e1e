"""Rotary positions on the GPU against the definition in 64 bits, within the
derived bounds of prompt_ref."""

import numpy as np
import pytest
import torch

from . import prompt_ref
from .gpu_util import say
from .prompt_ref import f64

pytestmark = pytest.mark.gpu
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
prompt = pytest.importorskip("paper_2608_28276_amd.prompt")
SENTINEL = -77.0


def tensor(seed, *shape, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * gain).to(torch.bfloat16).cuda()


def rope_of(D, first, rot, layout, scaling, magnitude=1.0):
    kw = dict(factor=4.0, original_len=4096, low_turns=1.0, high_turns=32.0)
    kind = dict(plain=0, linear=1, base=2, parts=3)[scaling]
    freq = prompt_ref.frequencies(rot, 1e4, scaling, 4.0, 4096, 1.0, 32.0)
    return prompt.make_rope(D, 1e4, rot_first=first, rot_dim=rot, layout=layout, scaling=kind, magnitude=magnitude,
                            **kw), freq


def compare(got, x, pos, live, freq, first, rot, layout, magnitude, what):
    """got [B, n, H, D] against x; rows that are not live keep the sentinel."""
    for b in range(x.shape[0]):
        m = live[b]
        want, tol = prompt_ref.rotate(f64(x[b, :m]), pos[b, :m], freq, first, rot, layout == 1, magnitude)
        err = np.abs(f64(got[b, :m]) - want)
        assert (err <= tol).all(), f"{what}: sequence {b}, worst {err.max()}"
        assert (f64(got[b, m:]) == SENTINEL).all(), f"{what}: rows behind sequence {b} written"


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("D, first, rot", [(128, 0, 128), (64, 0, 64), (192, 128, 64), (128, 0, 54), (128, 74, 54),
                                           (80, 0, 80), (128, 4, 64), (256, 0, 256), (6, 2, 2), (1024, 512, 256),
                                           (128, 8, 48), (96, 0, 8)])
@pytest.mark.parametrize("scaling", ["plain", "parts"])
def test_rotation(layout, D, first, rot, scaling):
    magnitude = 1.0 if scaling == "plain" else 1.139
    rope, freq = rope_of(D, first, rot, layout, scaling, magnitude)
    B, n, Hq, Hk = 3, 7, 5, 2
    q, k = tensor(1, B, n, Hq, D), tensor(2, B, n, Hk, D)
    start = torch.tensor([0, 130001, 2 ** 31 - 9], dtype=torch.int32).cuda()
    n_new = torch.tensor([7, 0, 3], dtype=torch.int32).cuda()
    q_out, k_out = torch.full_like(q, SENTINEL), torch.full_like(k, SENTINEL)
    say("rotation", layout, D, first, rot, scaling)
    prompt.rotate(rope, q, q_out, k, k_out, first=start, n_new=n_new)
    pos = start.cpu().numpy().astype(np.int64)[:, None] + np.arange(n)[None]
    for got, x in ((q_out, q), (k_out, k)):
        compare(got, x, pos, [7, 0, 3], freq, first, rot, layout, magnitude, "rotation")


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B, n, Hq, Hk", [(1, 1, 32, 8), (64, 1, 8, 1), (1, 5003, 3, 1), (5, 900, 2, 0), (2, 4, 0, 3)])
def test_sizes_and_positions(layout, B, n, Hq, Hk):
    D = 128
    rope, freq = rope_of(D, 0, D, layout, "linear")
    g = torch.Generator().manual_seed(B * 1000 + n)
    pos = torch.randint(-5, 1 << 20, (B, n), generator=g, dtype=torch.int32)
    say("sizes", layout, B, n, Hq, Hk)
    pairs = [(tensor(3, B, n, h, D), torch.full((B, n, h, D), SENTINEL, dtype=torch.bfloat16, device="cuda")) if h
             else (None, None) for h in (Hq, Hk)]
    prompt.rotate(rope, *pairs[0], *pairs[1], pos=pos.cuda())
    for x, y in pairs:
        if x is not None:
            compare(y, x, pos.numpy().astype(np.int64), [n] * B, freq, 0, D, layout, 1.0, "sizes")


@pytest.mark.parametrize("rot", [128, 64, 50])
@pytest.mark.parametrize("layout", [0, 1])
def test_in_place_equals_out_of_place_in_rows_of_a_projection(layout, rot):
    """Queries and keys rotated where a fused projection left them: the values and the rest of the rows untouched."""
    B, n, Hq, Hk, D = 2, 70, 4, 2, 128
    rope, _ = rope_of(D, 0, rot, layout, "plain")
    rows = tensor(5, B, n, (Hq + 2 * Hk) * D + 8)
    cut = lambda r, a, h: r[:, :, a * D:(a + h) * D].unflatten(2, (h, D))
    start = torch.tensor([11, 40000], dtype=torch.int32).cuda()
    n_new = torch.tensor([70, 33], dtype=torch.int32).cuda()
    q_out, k_out = (cut(rows, a, h).contiguous() for a, h in ((0, Hq), (Hq, Hk)))
    prompt.rotate(rope, cut(rows, 0, Hq), q_out, cut(rows, Hq, Hk), k_out, first=start, n_new=n_new)
    want = rows.clone()
    cut(want, 0, Hq).copy_(q_out)
    cut(want, Hq, Hk).copy_(k_out)
    prompt.rotate(rope, cut(rows, 0, Hq), cut(rows, 0, Hq), cut(rows, Hq, Hk), cut(rows, Hq, Hk), first=start, n_new=n_new)
    assert torch.equal(rows.view(torch.int16), want.view(torch.int16))


def test_unaligned_rows_equal_aligned_ones():
    """Rows that start off 16 bytes take the element-wise kernel: the same results bit for bit."""
    B, n, H, D = 2, 9, 3, 128
    rope, _ = rope_of(D, 0, 64, 0, "base")
    x = tensor(6, B, n, H, D)
    start = torch.tensor([5, 77777], dtype=torch.int32).cuda()
    want = torch.empty_like(x)
    prompt.rotate(rope, x, want, first=start)
    for shift, row in ((1, H * D), (0, H * D + 3)):
        room = torch.zeros(B * n * row + 1, dtype=torch.bfloat16, device="cuda")
        odd = room[shift:shift + B * n * row].view(B, n, row)[:, :, :H * D].unflatten(2, (H, D))
        odd.copy_(x)
        got = torch.empty_like(x)
        prompt.rotate(rope, odd, got, first=start)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
        prompt.rotate(rope, odd, odd, first=start)
        assert torch.equal(odd.contiguous().view(torch.int16), want.view(torch.int16))


def test_n_new_outside_its_range():
    rope, freq = rope_of(64, 0, 64, 0, "plain")
    x = tensor(7, 3, 4, 2, 64)
    out = torch.full_like(x, SENTINEL)
    prompt.rotate(rope, x, out, first=torch.zeros(3, dtype=torch.int32, device="cuda"),
                  n_new=torch.tensor([-3, 9, 4], dtype=torch.int32).cuda())
    compare(out, x, np.tile(np.arange(4), (3, 1)), [0, 4, 4], freq, 0, 64, 0, 1.0, "n_new")


def test_non_finite_elements_stay_in_their_pair():
    rope, _ = rope_of(128, 0, 128, 0, "plain")
    x = tensor(8, 1, 3, 1, 128)
    x[0, 1, 0, 5] = float("inf")
    x[0, 2, 0, 70] = float("nan")
    clean = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    out, want = torch.empty_like(x), torch.empty_like(x)
    first = torch.zeros(1, dtype=torch.int32, device="cuda")
    prompt.rotate(rope, x, out, first=first)
    prompt.rotate(rope, clean, want, first=first)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[0, 1, 0, [5, 69]] = True
    hit[0, 2, 0, [6, 70]] = True
    assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any()


def test_caller_frequencies_and_another_stream():
    rope, _ = rope_of(64, 0, 64, 1, "plain")
    freq = np.linspace(0.0, 3.0, 32)
    for i, f in enumerate(freq):
        rope.turns[i] = f / (2 * np.pi)
    x = tensor(9, 1, 20, 3, 64)
    out = torch.full_like(x, SENTINEL)
    pos = torch.arange(20, dtype=torch.int32, device="cuda").view(1, 20) * 1000
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        prompt.rotate(rope, x, out, pos=pos)
    s.synchronize()
    compare(out, x, pos.cpu().numpy().astype(np.int64), [20], freq, 0, 64, 1, 1.0, "caller's frequencies")


def test_graph_replays_follow_the_positions():
    rope, freq = rope_of(128, 0, 128, 0, "plain")
    x, out = tensor(10, 2, 5, 4, 128), torch.empty(2, 5, 4, 128, dtype=torch.bfloat16, device="cuda")
    first = torch.tensor([0, 9], dtype=torch.int32).cuda()
    prompt.rotate(rope, x, out, first=first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prompt.rotate(rope, x, out, first=first)
    for step in range(3):
        first += 123
        out.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        pos = first.cpu().numpy().astype(np.int64)[:, None] + np.arange(5)[None]
        compare(out, x, pos, [5, 5], freq, 0, 128, 0, 1.0, f"replay {step}")


def test_refusals_of_tensors():
    rope, _ = rope_of(128, 0, 128, 0, "plain")
    x = tensor(11, 2, 3, 4, 128)
    first = torch.zeros(2, dtype=torch.int32, device="cuda")

    def status(*args, **kw):
        with pytest.raises(pask.PaskError) as e:
            prompt.rotate(rope, *args, **kw)
        return e.value.status

    ARG, SHAPE = pask.PASK_E_ARG, pask.PASK_E_SHAPE
    assert status(x.float(), x, first=first) == ARG
    assert status(x, x.cpu(), first=first) == ARG
    assert status(x, x[:1], first=first) == SHAPE
    assert status(x, x[:, :, :2], first=first) == SHAPE        # another number of heads
    assert status(x[..., :64], x[..., :64], first=first) == SHAPE
    assert status(x.transpose(1, 2), x, first=first) == ARG
    assert status(x.transpose(2, 3).contiguous().transpose(2, 3), x, first=first) == ARG
    assert status(x, x, first=first.long()) == ARG
    assert status(x, x, first=first[:1]) == SHAPE
    assert status(x, x, first=first, pos=first) == SHAPE
    assert status(x, x) == ARG
    assert status(x, x, first=first, n_new=first[:1]) == SHAPE
    assert status(x, x, first=first, first_stride=0) == ARG
    assert status(x, None, first=first) == ARG
    assert status(x.expand(2, 3, 4, 128)[:1].expand(2, 3, 4, 128), x, first=first) == ARG
