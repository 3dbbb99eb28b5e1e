"""Partial results of the keys' pieces: what the joining reads was written by
this call, also where pieces are empty and rows are not there, and calls of more
pieces than a round of the joining takes."""

import numpy as np
import pytest
import torch

from . import prompt_ref
from .gpu_util import say
from .latent_ref import check
from .prompt_ref import f64

pytestmark = pytest.mark.gpu
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
prompt = pytest.importorskip("paper_2608_28276_amd.prompt")
from .test_gpu_prompt import MIXED, SENTINEL, Run, normal  # noqa: E402

CANARY = 4096


def pieces_of(geom, batch, max_q, hint):
    """From the workspace: an output, a reference and a sum for each row and piece."""
    need = prompt.pask_prompt_workspace_bytes(geom, batch, max_q, hint)
    return need, need // (batch * geom.n_q_heads * max_q * (geom.head_dim + 2) * 4)


# pieces: of 32 rows in more and in fewer than the 8 that one wave joins, of 256 rows; lengths far below the hint
@pytest.mark.parametrize("Hq, Hkv, max_q, lens, n_q, hint, least, most", [
    (8, 2, 3, [3000, 40, 0, 1, 700], [3, 0, 0, 1, 2], 30000, 9, 512),
    (8, 2, 8, [500, 17, 90], [8, 0, 5], 512, 2, 8),
    (8, 1, 100, [1500, 3, 100], [100, 0, 33], 30000, 9, 512),
    (8, 8, 70, [600, 70], [70, 1], 2000, 2, 8),
])
@pytest.mark.parametrize("D", [64, 128])
def test_nothing_is_read_from_the_workspace_that_the_call_did_not_write(D, Hq, Hkv, max_q, lens, n_q, hint, least, most):
    B = len(lens)
    r = Run(B, Hq, Hkv, D, 30000, MIXED, window=11, seed=D + max_q, pages=600)
    r.append(lens)
    need, pieces = pieces_of(r.s.geom, B, max_q, hint)
    say("workspace", D, Hq, Hkv, max_q, "pieces", pieces, "bytes", need)
    assert least <= pieces <= most
    q = normal(r.gen, B, max_q, Hq, D)
    counts = torch.tensor(n_q, dtype=torch.int32).cuda()
    bits = []
    for fill in (0x00, 0xFF, 0x7F):
        ws = torch.full((need + CANARY,), fill, dtype=torch.uint8, device="cuda")
        ws[need:] = 0x5A
        out = torch.full((B, max_q, Hq, D), SENTINEL, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((B, max_q, Hq), SENTINEL, device="cuda")
        prompt.pask_prompt_attn(r.s.cache, 0, B, max_q, counts, None, q.cuda(), out, lse, r.s.softmax_scale, hint, ws, need,
                                r.s.stream)
        torch.cuda.synchronize()
        assert (ws[need:] == 0x5A).all(), "written behind the workspace"
        bits.append((out.view(torch.int16).cpu(), lse.view(torch.int32).cpu()))
    assert all(torch.equal(x, y) for b in bits[1:] for x, y in zip(bits[0], b))
    for b, n in enumerate(n_q):
        want, want_lse, tol, lse_tol = prompt_ref.prompt(r.ref, b, f64(q[b, :n]), r.ref.n_pos(b) - n, r.s.softmax_scale)
        check(f64(out[b, :n]), want, tol, f"out of sequence {b}")
        check(f64(lse[b, :n]), want_lse, lse_tol, f"lse of sequence {b}")
        assert (out[b, n:] == SENTINEL).all() and (lse[b, n:] == SENTINEL).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [40000, 4100])
def test_more_pieces_than_a_round_of_the_joining(D, n):
    """One sequence, one KV head, 70,000 tokens foreseen: 512 pieces of what is there, four waves 256 of them a round."""
    r = Run(1, 4, 1, D, 70000, MIXED, window=21, seed=n, pages=n // 16 + 2)
    need, pieces = pieces_of(r.s.geom, 1, 3, 70000)
    assert pieces == 512
    r.append([n])
    r.attend([3], what="pieces")
    r.attend([3], first=[n // 2], what="pieces, in the middle")


@pytest.mark.parametrize("Hq, Hkv, n_q, n", [(8, 2, 3, 40), (8, 2, 3, 1900), (8, 8, 100, 300), (8, 1, 100, 2900)])
def test_outputs_may_take_the_queries_place(Hq, Hkv, n_q, n):
    """Few and many rows, with one piece and with more: a workgroup writes rows that it alone reads, after reading them."""
    r = Run(2, Hq, Hkv, 128, 3000, MIXED, window=9, seed=n + n_q)
    r.append([n, n // 2 + n_q])
    q = normal(r.gen, 2, n_q, Hq, 128).cuda()
    out = torch.empty_like(q)
    r.s.prompt(0, q, out, max_ctx_hint=n)
    r.s.prompt(0, q, q, max_ctx_hint=n)
    assert torch.equal(q.view(torch.int16), out.view(torch.int16))
