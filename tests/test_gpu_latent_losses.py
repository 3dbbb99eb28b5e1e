"""Full pools and full sequences, exactly: which flag is set by which kernel, what is counted, what stays."""

import numpy as np
import pytest
import torch

from .latent_ref import DROP, HIGH, LOW
from .test_gpu_latent import DEV, Pair, pask

pytestmark = pytest.mark.gpu


def add(p, kind, tokens):
    """One token per sequence through the bulk call, the one-token call or a decode step; the reference is not told."""
    tags, c, r = (x.to(DEV) for x in tokens)
    if kind == "bulk":
        p.sess.append(0, tags, c, r, n_new=torch.ones(p.batch, dtype=torch.int32, device=DEV))
    elif kind == "one":
        p.sess.append(0, tags, c, r)
    else:
        q = p.queries()
        out = torch.empty(p.batch, p.heads, p.rank, dtype=torch.bfloat16, device=DEV)
        lse = torch.empty(p.batch, p.heads, device=DEV)
        p.sess.decode(0, q.to(DEV), out, lse, tags[:, 0].contiguous(), c[:, 0].contiguous(), r[:, 0].contiguous())
        return q, out, lse
    return None


@pytest.mark.parametrize("kind", ["bulk", "one", "step"])
@pytest.mark.parametrize("action, flag", [(HIGH, "PASK_FLAG_HI_POOL_EXHAUSTED"), (LOW, "PASK_FLAG_LO_POOL_EXHAUSTED")])
def test_a_full_pool(action, flag, kind):
    """Both pools have two pages; the tokens of one action fill the one's exactly, or all but six slots of it."""
    p = Pair(batch=2, heads=5, rank=128, rope=32, max_tokens=64, hi_pages=2, lo_pages=2, action=[action], floor=[DROP],
             seed=action)
    z = lambda n: (torch.zeros(2, n, dtype=torch.uint8),) + p.tokens(n)[1:]
    p.append([16, 10], tokens=z(16))
    assert p.sess.stats()[1] == pask.PASK_OK
    t = z(1)                                         # sequence 0 needs a third page, sequence 1 has room
    seen = add(p, kind, t)
    lost = np.array([1, 0])

    def check():
        st, status = p.sess.stats()
        assert status == pask.PASK_E_DEVICE_FLAG and st.device_flags == getattr(pask, flag)
        want = p.ref.cnt.copy()
        want[:, 2] += lost                           # a lost token has its position
        want[:, 5] += lost
        assert p.sess.counters()[:, 0, :6].cpu().numpy().tolist() == want.tolist()
        assert st.n_lost == lost.sum() and (st.n_high, st.n_low) == tuple(want[:, :2].sum(0))
        assert (st.hi_pages_used, st.lo_pages_used) == ((2, 0) if action == HIGH else (0, 2))
        assert (p.sess.buf[p.sess.nbytes:] == 0xFF).all()
        p.check_read()
        if seen:
            p.check_attention(*seen)

    p.ref.append(1, [0], *(x[1].double().numpy() for x in t[1:]))
    check()
    for _ in range(5):
        t = z(1)
        seen = add(p, kind, t)
        p.ref.append(1, [0], *(x[1].double().numpy() for x in t[1:]))
        lost[0] += 1
    check()                                          # both sequences' pages are full now
    seen = add(p, kind, z(1))
    lost += 1
    check()
    tags, c, r = z(20)                               # many at once
    p.sess.append(0, tags.to(DEV), c.to(DEV), r.to(DEV))
    lost += 20
    seen = None
    check()


@pytest.mark.parametrize("kind", ["bulk", "one", "step"])
def test_a_full_sequence(kind):
    """The sequence's last position is kept; what comes after has none: lost, of the flag of its own."""
    p = Pair(batch=2, heads=5, rank=128, rope=32, max_tokens=20, action=[HIGH, LOW], floor=[DROP, DROP], seed=9)
    p.append([19, 20])
    add(p, kind, t := p.tokens(1))
    p.ref.append(0, t[0][0].tolist(), *(x[0].double().numpy() for x in t[1:]))
    p.ref.append(1, t[0][1].tolist(), *(x[1].double().numpy() for x in t[1:]))
    st, status = p.sess.stats()
    assert status == pask.PASK_E_DEVICE_FLAG and st.device_flags == pask.PASK_FLAG_SEQ_CAPACITY and st.n_lost == 1
    p.check_counters()
    p.check_read()


@pytest.mark.parametrize("kind", ["bulk", "one", "step"])
def test_a_tag_outside_the_table(kind):
    """Kept HIGH as a forced entry, and flagged."""
    p = Pair(batch=2, heads=5, rank=128, rope=32, action=[LOW, DROP], floor=[DROP, DROP], seed=10)
    p.append([5, 6])
    assert p.sess.stats()[1] == pask.PASK_OK
    tags, c, r = p.tokens(1)
    tags[:] = torch.tensor([[0], [2]], dtype=torch.uint8)
    add(p, kind, (tags, c, r))
    for b in range(2):
        p.ref.append(b, tags[b].tolist(), c[b].double().numpy(), r[b].double().numpy())
    st, status = p.sess.stats()
    assert status == pask.PASK_E_DEVICE_FLAG and st.device_flags == pask.PASK_FLAG_BAD_TAG and st.n_lost == 0
    p.check_counters()
    p.check_read()


@pytest.mark.parametrize("kind", ["bulk", "one", "step"])
@pytest.mark.parametrize("action", [HIGH, LOW])
def test_a_pool_full_for_long(action, kind):
    """However many tokens a full pool has lost, its first page is not handed out again."""
    p = Pair(batch=2, heads=5, rank=128, rope=32, max_tokens=64, hi_pages=2, lo_pages=2, action=[action], floor=[DROP],
             seed=action + 20)
    z = lambda n: (torch.zeros(2, n, dtype=torch.uint8),) + p.tokens(n)[1:]
    p.append([16, 16], tokens=z(16))
    at = p.sess.layout.status_off + 8 + 4 * (action == LOW)
    cursor = p.sess.buf[at:at + 4].view(torch.int32)
    cursor.fill_(-2)                                 # as after 2^32 - 4 tokens that found no page
    for _ in range(3):
        seen = add(p, kind, z(1))
    st, status = p.sess.stats()
    assert status == pask.PASK_E_DEVICE_FLAG and st.n_lost == 6 and st.n_high + st.n_low == 32
    assert (st.hi_pages_used, st.lo_pages_used) == ((2, 0) if action == HIGH else (0, 2))
    p.check_read()
    if seen:
        p.check_attention(*seen)
