"""int4 pages that hold scales above 2728 beside small ones: neither a wide
entry that a query does not see nor the wide groups of one that it sees take
bits from the others.  The bounds are latent_ref's with prompt_ref's 2^-33 for
the weights, and nothing for the size of what else a page holds: a LOW key is
exact and a LOW value is rounded by 2^-11 of itself at most (an int4 code times
an fp16 scale is a multiple of fp16's smallest step, so it is exact below fp16's
normal range)."""

import numpy as np
import pytest
import torch

from . import latent_ref
from .gpu_util import say
from .latent_ref import check
from .prompt_ref import LOW, f64

pytestmark = pytest.mark.gpu
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
from .test_gpu_prompt import Run, normal  # noqa: E402

WIDE = 4.0e5                                          # of an element: a scale of 57,000
N, NEW = 211, 13


def attend(r, q, first, what):
    """One call over the cache of sequence 0, checked row by row within the bounds of what each row sees."""
    n, hq, d = q.shape
    out = torch.full((1, n, hq, d), -77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((1, n, hq), -77.0, device="cuda")
    say("attend", what, "n", n, "D", d, "first", first)
    r.s.prompt(0, q[None].cuda(), out, lse, first=torch.tensor([first], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    pos, k, v = r.ref.visible(0)
    seen = pos[None] <= first + np.arange(n)[:, None]
    for h in range(hq):
        g = h * k.shape[1] // hq
        want, want_lse, tol, lse_tol = latent_ref.attention(f64(q[:, h]), k[:, g], v[:, g], r.s.softmax_scale, seen)
        tol += 2.0 ** -33 * (seen @ np.abs(v[:, g]))
        check(f64(out[0, :, h]), want, tol, f"{what}: out of head {h}")
        check(f64(lse[0, :, h]), want_lse, lse_tol, f"{what}: lse of head {h}")


def small_and_wide(gen, n, D, where, all_groups):
    """[1, n, 2, D] of about 2^-14, at tokens `where` of WIDE's size, in all 32-element groups or the first one."""
    x = normal(gen, 1, n, 2, D, gain=2.0 ** -14)
    x[:, where, :, :D if all_groups else 32] *= WIDE * 2.0 ** 12
    return x


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [3, 150])
@pytest.mark.parametrize("what", ["keys", "values"])
def test_hidden_wide_entries_take_no_bits_from_what_is_seen(D, n_q, what):
    """The last tokens are wide and behind every query; they share pages, and the units of two pages, with seen ones."""
    r = Run(1, 4, 2, D, 400, (LOW,), seed=D + n_q)
    where = torch.arange(N - NEW, N)
    x = small_and_wide(r.gen, N, D, where, True)
    r.append([N], **({"k": x} if what == "keys" else {"v": x}))
    r.s.softmax_scale = 2.0 ** 11 if what == "keys" else 0.1
    for back in (0, 1, 5):
        attend(r, normal(r.gen, n_q, 4, D), N - NEW - n_q - back, what)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [3, 150])
def test_wide_groups_beside_small_ones_of_the_same_keys(D, n_q):
    """Every fifth key is wide in its first group, where the queries are 0: the others' scores are exact."""
    r = Run(1, 4, 2, D, 400, (LOW,), seed=D + n_q + 1)
    r.append([N], k=small_and_wide(r.gen, N, D, torch.arange(2, N, 5), False))
    r.s.softmax_scale = 2.0 ** 11
    q = normal(r.gen, n_q, 4, D)
    q[:, :, :32] = 0.0
    attend(r, q, N - n_q, "keys' groups")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [3, 150])
@pytest.mark.parametrize("group", [0, 1])
def test_wide_groups_beside_small_ones_of_the_same_values(D, n_q, group):
    """Every fifth value, and whole pages of them, are wide in one group: the other groups' outputs are about 2^-16."""
    r = Run(1, 4, 2, D, 400, (LOW,), seed=D + n_q + 2 + group)
    where = torch.cat([torch.arange(2, 100, 5), torch.arange(112, 160), torch.tensor([N - 1])])
    v = normal(r.gen, 1, N, 2, D, gain=2.0 ** -14)
    v[:, where, :, 32 * group:32 * group + 32] *= WIDE * 2.0 ** 12
    r.append([N], v=v)
    r.s.softmax_scale = 0.1
    attend(r, normal(r.gen, n_q, 4, D), N - n_q, "values' groups")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [4, 150])
def test_wide_keys_that_are_seen_are_exact(D, n_q):
    """Keys of every size in one page, all of them seen: scores within the bound of fp32 sums."""
    r = Run(1, 4, 2, D, 400, (LOW,), seed=D + n_q + 5)
    k = normal(r.gen, 1, N, 2, D)
    k *= 2.0 ** torch.randint(-14, 18, (1, N, 2, D // 32), generator=r.gen).repeat_interleave(32, 3)
    r.append([N], k=k.to(torch.bfloat16))
    r.s.softmax_scale = 2.0 ** -15
    attend(r, normal(r.gen, n_q, 4, D), N - n_q, "keys of every size")
