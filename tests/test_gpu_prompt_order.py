"""Calls whose workgroups take turns begin with the longest sequences: more of
them than compute units, in batches that are ranked (up to 64) and not (above)."""

import pytest

from .test_gpu_prompt import MIXED, Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B, n_q", [(64, 3), (65, 3), (64, 20), (66, 20), (40, 11)])
def test_ragged_batches_in_turns(B, n_q):
    r = Run(B, 32, 8, 64, 400, MIXED, window=7, seed=B + n_q)
    lens = [(37 * b * b) % 390 for b in range(B)]     # equal lengths, empty sequences among them
    r.append(lens)
    r.attend([min(n_q, n) for n in lens], max_q=n_q, what="turns")
