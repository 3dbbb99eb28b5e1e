"""The largest calls of the latent entry points, on the host (no GPU): refused before anything is launched."""

import pytest

from .test_latent_host import A, fake_cache, geom, latent, pask, policy, status


@pytest.mark.parametrize("n", [2 ** 28 - 60, 2 ** 28])
@pytest.mark.parametrize("n_new", [0, A])
def test_append_of_more_pages_than_a_launch_fills(n, n_new):
    """Refused as a whole: launched, the tokens would be counted and their pages never written."""
    c = fake_cache(geom(max_batch=1, rank=128, rope_dim=32, max_tokens_per_seq=2 ** 28))
    assert status(latent.pask_latent_append, policy(), c, 0, 1, n_new, n, A, A, A) == pask.PASK_E_SHAPE
