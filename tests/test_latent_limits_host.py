"""The largest calls of the entry points that append, on the host (no GPU): refused before anything is launched."""

import pytest

from .test_latent_host import A, fake_cache, geom, latent, pask, policy, status


@pytest.mark.parametrize("n", [2 ** 28 - 60, 2 ** 28])
@pytest.mark.parametrize("n_new", [0, A])
def test_append_of_more_pages_than_a_launch_fills(n, n_new):
    """Refused as a whole: launched, the tokens would be counted and their pages never written."""
    c = fake_cache(geom(max_batch=1, rank=128, rope_dim=32, max_tokens_per_seq=2 ** 28))
    assert status(latent.pask_latent_append, policy(), c, 0, 1, n_new, n, A, A, A) == pask.PASK_E_SHAPE


@pytest.mark.parametrize("n, n_new, window", [(2 ** 28 - 60, 0, 0), (2 ** 28, A, 0), (2 ** 28 - 100, 0, 40),
                                              (1, A, 2 ** 28 - 61), (2 ** 24, 0, 2 ** 24)])
def test_grouped_query_append_of_more_pages_than_a_launch_fills(n, n_new, window):
    g = pask.make_geom(max_batch=1, n_layers=2, n_q_heads=1, n_kv_heads=1, head_dim=64, max_tokens_per_seq=2 ** 28,
                       hi_pages=40, lo_pages=30, recent_window=window)
    c = pask.pask_cache()
    c.geom, c.base, c.bytes = g, 1 << 40, pask.pask_cache_bytes(g)
    assert c.bytes > 0
    assert status(pask.pask_kv_append, policy(window=window), c, 0, 1, n_new, n, A, A, A) == pask.PASK_E_SHAPE
