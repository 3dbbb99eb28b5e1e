"""Rotations of so many rows that a workgroup takes four or eight of them at a
turn (4,096 and 16,384 rows), in each of the three forms: whole 16-byte chunks,
heads through LDS, element by element."""

import numpy as np
import pytest
import torch

from .gpu_util import say
from .test_gpu_rope import SENTINEL, compare, prompt, rope_of

pytestmark = pytest.mark.gpu

# head_dim, first rotated, rotated, elements that the rows are off 16 bytes by
FORMS = {"chunks": (64, 0, 64, 0), "part in chunks": (96, 32, 48, 0), "staged": (64, 6, 50, 0), "elements": (64, 0, 64, 1),
         "elements of odd heads": (10, 2, 6, 0)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B, n", [(5, 900), (3, 1367), (17, 1001)])
@pytest.mark.parametrize("in_place", [False, True])
def test_several_rows_a_workgroup(form, layout, B, n, in_place):
    D, first, rot, off = FORMS[form]
    Hq, Hk = 3, 1
    rope, freq = rope_of(D, first, rot, layout, "parts", 1.139)
    g = torch.Generator().manual_seed(B + n + D)
    room = torch.randn(B * n * (Hq + Hk) * D + 8, generator=g).to(torch.bfloat16).cuda()
    rows = room[off:off + B * n * (Hq + Hk) * D].view(B, n, (Hq + Hk) * D)
    cut = lambda t, a, h: t[:, :, a * D:(a + h) * D].unflatten(2, (h, D))
    live = [(b * 613 + n // 3) % (n + 1) for b in range(B)]
    live[1], live[2] = 0, n
    start = torch.randint(0, 1 << 20, (B,), generator=g, dtype=torch.int32)
    say("rows", form, layout, B, n, "in place" if in_place else "")
    before = rows.clone()
    if in_place:
        outs = [cut(rows, 0, Hq), cut(rows, Hq, Hk)]
    else:
        outs = [torch.full((B, n, h, D), SENTINEL, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hk)]
    prompt.rotate(rope, cut(rows, 0, Hq), outs[0], cut(rows, Hq, Hk), outs[1], first=start.cuda(),
                  n_new=torch.tensor(live, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    pos = start.numpy().astype(np.int64)[:, None] + np.arange(n)[None]
    for out, a, h in ((outs[0], 0, Hq), (outs[1], Hq, Hk)):
        x = cut(before, a, h)
        if in_place:                                  # rows that are not live keep what they held
            for b in range(B):
                assert torch.equal(out[b, live[b]:].view(torch.int16), x[b, live[b]:].view(torch.int16))
            out = out.clone()
            for b in range(B):
                out[b, live[b]:] = SENTINEL
        compare(out, x, pos, live, freq, first, rot, layout, 1.139, form)
    if not in_place:
        assert torch.equal(rows.view(torch.int16), before.view(torch.int16))
