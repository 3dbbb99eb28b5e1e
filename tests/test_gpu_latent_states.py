"""Going back to saved states of a latent session: what is valid comes back exactly, what is void is refused."""

import pytest
import torch

from .latent_ref import HIGH, LOW
from .test_gpu_latent import DEV, Pair, pask

pytestmark = pytest.mark.gpu


def refused(sess, state):
    before = sess.buf.clone()
    with pytest.raises(pask.PaskError) as e:
        sess.restore(state)
    assert e.value.status == pask.PASK_E_ARG
    assert torch.equal(sess.buf, before)


def extra(p, n):
    """n tokens that the reference is not told of."""
    for _ in range(n):
        tags, c, r = p.tokens(1)
        p.sess.append(0, tags.to(DEV), c.to(DEV), r.to(DEV))


def test_going_back_voids_the_states_after():
    """Saved, appended, saved again, gone back and appended: the second state's pages hold the new tokens."""
    p = Pair(batch=2, heads=4, rank=128, rope=32, seed=1, action=[HIGH, LOW], floor=[HIGH, LOW])
    p.append([20, 15])
    first = p.sess.save()
    extra(p, 20)
    second = p.sess.save()
    extra(p, 3)
    third = p.sess.save()
    p.sess.restore(second)                           # in order: valid
    refused(p.sess, third)
    p.sess.restore(first)
    p.check_counters()
    p.append([18, 30])
    refused(p.sess, second)
    p.check_counters()
    p.check_read()


def test_branches_from_one_state():
    """A state is gone back to again and again; newer states of a branch are valid until then."""
    p = Pair(batch=3, heads=4, rank=128, rope=32, seed=2)
    p.append([40, 16, 15])
    root = p.sess.save()
    for k in range(1, 4):
        p.sess.restore(root)
        extra(p, 7 * k)
        tip = p.sess.save()
        extra(p, 20)
        want = tip._head.clone()
        p.sess.restore(tip)
        assert torch.equal(p.sess._head(), want)
    p.sess.restore(root)
    refused(p.sess, tip)
    p.append([33, 1, 20])
    p.check_counters()
    p.check_read()
    p.decode(p.queries())


def test_a_reset_voids_every_state():
    p = Pair(batch=2, heads=4, rank=128, rope=32, seed=3)
    p.append([20, 30])
    states = [p.sess.save(), p.sess.save()]
    p.sess.reset()
    for s in states:
        refused(p.sess, s)
    assert p.sess.counters()[..., :6].eq(0).all()


def test_other_things_are_refused():
    """Another session's state names pages that this one never wrote; a tensor says nothing of where it is from."""
    p, q = (Pair(batch=2, heads=4, rank=128, rope=32, seed=s) for s in (4, 5))
    p.append([20, 30])
    state = p.sess.save()
    for x in (state, state._head, None):
        refused(q.sess, x)
    p.sess.restore(state)
    p.check_counters()
    p.check_read()


def test_states_that_nobody_holds_are_let_go():
    p = Pair(batch=2, heads=4, rank=128, rope=32, seed=6)
    for _ in range(5):
        p.sess.save()
    assert len(p.sess._saved) == 0


def test_a_state_of_a_capture_stays_in_it():
    """A step tried and taken back in a graph leaves the cache as it was at each replay; outside, the captured state is
    refused (before a replay its memory holds nothing)."""
    p = Pair(batch=2, heads=4, rank=128, rope=32, seed=7)
    p.append([20, 30])
    tags, c, r = (x.to(DEV) for x in p.tokens(1))
    outer = p.sess.save()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        state = p.sess.save()
        p.sess.append(0, tags, c, r)
        p.sess.restore(state)
    refused(p.sess, state)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        p.check_counters()
        refused(p.sess, state)
        p.append([1, 3])                             # eager work between
        p.check_read()
    extra(p, 2)
    p.sess.restore(outer)
    assert p.sess.counters()[:, 0, 2].tolist() == [20, 30]
