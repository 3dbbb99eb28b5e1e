"""Prompts over keys at given positions, on the host (no GPU): the refusals, none of which may reach a HIP call."""

import pytest

from .test_latent_host import A, PROMPT, latent, pask, status

POS = dict(PROMPT, pos=A, q_first=A)


@pytest.mark.parametrize("want, over", [
    ("PASK_E_ARG", dict(pos=0)), ("PASK_E_ARG", dict(pos=A + 2)), ("PASK_E_ARG", dict(q_first=0)),
    ("PASK_E_ARG", dict(q_first=A + 1)), ("PASK_E_ARG", dict(max_q=0, q_first=0)), ("PASK_E_SHAPE", dict(batch=0)),
    ("PASK_E_SHAPE", dict(n_heads=129)), ("PASK_E_SHAPE", dict(nope_dim=96)), ("PASK_E_ARG", dict(max_q=-1)),
    ("PASK_E_ARG", dict(cu_q=0)), ("PASK_E_ARG", dict(cu_k=A + 2)), ("PASK_E_ARG", dict(q=0)),
    ("PASK_E_ARG", dict(kv=A + 8)), ("PASK_E_ARG", dict(out=0)), ("PASK_E_ARG", dict(lse=A + 1)),
    ("PASK_E_ARG", dict(softmax_scale=float("inf"))),
    ("PASK_E_SHAPE", dict(batch=65535, n_heads=128, max_q=1000, total_q=1 << 30))])
def test_refusals(want, over):
    assert status(latent.pask_latent_prompt_attn_pos, **dict(POS, **over)) == getattr(pask, want)


@pytest.mark.parametrize("over", [dict(max_q=0), dict(total_q=0, q=0, out=0), dict(max_q=0, total_k=0, pos=0)])
def test_no_query_is_no_call(over):
    latent.pask_latent_prompt_attn_pos(**dict(POS, **over))
