"""The entry points of pask_prompt.h on the host (no GPU): exports, rotary
frequencies, workspace sizes and every refusal, none of which may reach a HIP
call."""

import ctypes as C
import math
import os
import re

import numpy as np
import pytest
import torch

from . import prompt_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
prompt = pytest.importorskip("paper_2608_28276_amd.prompt")
AT = 1 << 20                                          # an address that nothing may touch


def geom(**kw):
    d = dict(max_batch=4, n_layers=2, n_q_heads=16, n_kv_heads=4, head_dim=128, max_tokens_per_seq=5000, hi_pages=40,
             lo_pages=30, recent_window=0)
    d.update(kw)
    return pask.make_geom(**d)


def fake_cache(g=None, at=AT):
    c = pask.pask_cache()
    c.geom = g or geom()
    c.base = at
    c.bytes = pask.pask_cache_bytes(c.geom)
    return c


def status(f, *args, **kw):
    with pytest.raises(pask.PaskError) as e:
        f(*args, **kw)
    return e.value.status


def test_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "pask_prompt.h")).read()
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(pask_\w+)\s*\(", text, re.M))
    assert names == set(prompt.EXPORTS)
    for n in names:
        assert hasattr(pask.library(), n) and hasattr(prompt, n), n
    for n in ("PASK_ROPE_MAX_PAIRS", "PASK_ROPE_MAX_HEAD_DIM", "PASK_ROPE_MAX_HEADS"):
        assert int(re.search(rf"#define {n} (\d+)", text).group(1)) == getattr(prompt, n)


@pytest.mark.parametrize("rot", [2, 6, 64, 128, 256])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "parts"])
def test_frequencies(rot, scaling):
    kind = dict(plain=0, linear=1, base=2, parts=3)[scaling]
    r = prompt.make_rope(256, 5e5, rot_dim=rot, scaling=kind, factor=3.5, original_len=4096, low_turns=1.0,
                         high_turns=16.0, magnitude=1.25)
    want = prompt_ref.frequencies(rot, 5e5, scaling, 3.5, 4096, 1.0, 16.0) / (2 * math.pi)
    got = np.array(r.turns[:rot // 2])
    assert np.allclose(got, want, rtol=1e-14, atol=0)
    assert all(x == 0.0 for x in r.turns[rot // 2:]) and r.magnitude == 1.25
    if scaling == "base" and rot > 2:                 # the slowest pair ends up factor times slower
        assert math.isclose(got[-1] * 3.5, 5e5 ** (-(rot - 2) / rot) / (2 * math.pi), rel_tol=1e-12)


@pytest.mark.parametrize("bad, want", [
    (dict(head_dim=1), "SHAPE"), (dict(head_dim=1026), "SHAPE"), (dict(rot_dim=0), "SHAPE"), (dict(rot_dim=63), "SHAPE"),
    (dict(rot_dim=258, head_dim=1024), "SHAPE"), (dict(rot_first=-2), "SHAPE"), (dict(rot_first=66, rot_dim=64), "SHAPE"),
    (dict(layout=2), "ARG"), (dict(layout=-1), "ARG"), (dict(scaling=4), "ARG"), (dict(scaling=-1), "ARG"),
    (dict(base=0.0), "ARG"), (dict(base=-1.0), "ARG"), (dict(base=math.inf), "ARG"), (dict(base=math.nan), "ARG"),
    (dict(base=5e-324, rot_dim=128), "ARG"), (dict(magnitude=math.nan), "ARG"), (dict(scaling=1, factor=0.5), "ARG"),
    (dict(scaling=2, factor=math.inf), "ARG"), (dict(scaling=3, factor=math.nan), "ARG"),
    (dict(scaling=3, original_len=0), "ARG"), (dict(scaling=3, low_turns=-1.0), "ARG"),
    (dict(scaling=3, low_turns=4.0, high_turns=4.0), "ARG"), (dict(scaling=3, high_turns=math.inf), "ARG"),
    (dict(scaling=3, low_turns=math.nan), "ARG")])
def test_rope_refusals(bad, want):
    kw = dict(head_dim=128, base=1e4)
    kw.update(bad)
    assert status(prompt.make_rope, kw.pop("head_dim"), kw.pop("base"), **kw) == getattr(pask, "PASK_E_" + want)


def test_rope_ignores_what_its_scaling_does_not_read():
    r = prompt.make_rope(64, 1e4, factor=math.nan, original_len=-5, low_turns=9.0, high_turns=1.0)
    assert r.turns[0] == 1 / (2 * math.pi)
    assert prompt._lib.pask_rope_init(None, 64, 0, 64, 0, 1e4, 0, 1.0, 1, 1.0, 32.0, 1.0) == pask.PASK_E_ARG


def apply_args(**kw):
    d = dict(rope=prompt.make_rope(128), batch=2, max_new=3, n_new=None, first=AT, first_stride=1, pos=None, n_q_heads=4,
             q_in=AT, q_in_stride=512, q_out=2 * AT, q_out_stride=512, n_k_heads=2, k_in=3 * AT, k_in_stride=256,
             k_out=4 * AT, k_out_stride=256)
    d.update(kw)
    return d


@pytest.mark.parametrize("bad, want", [
    (dict(batch=-1), "SHAPE"), (dict(max_new=-1), "SHAPE"), (dict(batch=1 << 16, max_new=1 << 15), "SHAPE"),
    (dict(n_q_heads=-1), "SHAPE"), (dict(n_k_heads=1025, k_in_stride=1 << 20, k_out_stride=1 << 20), "SHAPE"),
    (dict(first=None), "ARG"), (dict(pos=AT), "ARG"), (dict(first=None, pos=AT + 2), "ARG"), (dict(first=AT + 1), "ARG"),
    (dict(n_new=AT + 2), "ARG"), (dict(q_in=None), "ARG"), (dict(q_out=None), "ARG"), (dict(k_in=AT + 1), "ARG"),
    (dict(k_out=AT + 1), "ARG"), (dict(q_in_stride=511), "ARG"), (dict(q_out_stride=0), "ARG"),
    (dict(first_stride=-1), "ARG"), (dict(k_in_stride=-256), "ARG"), (dict(k_out_stride=1 << 41), "ARG"),
    (dict(q_out=AT, q_out_stride=520), "ARG")])
def test_apply_refusals(bad, want):
    assert status(prompt.pask_rope_apply, **apply_args(**bad)) == getattr(pask, "PASK_E_" + want)


@pytest.mark.parametrize("field, value", [("head_dim", 0), ("rot_first", 1), ("rot_dim", 3), ("rot_dim", 300),
                                          ("layout", 7), ("magnitude", math.inf)])
def test_apply_refuses_a_broken_rope(field, value):
    r = prompt.make_rope(128)
    setattr(r, field, value)
    assert status(prompt.pask_rope_apply, **apply_args(rope=r)) == pask.PASK_E_ARG
    r = prompt.make_rope(128)
    r.turns[63] = math.nan
    assert status(prompt.pask_rope_apply, **apply_args(rope=r)) == pask.PASK_E_ARG


def test_apply_of_nothing_is_ok():
    prompt.pask_rope_apply(**apply_args(batch=0))
    prompt.pask_rope_apply(**apply_args(max_new=0))
    prompt.pask_rope_apply(**apply_args(n_q_heads=0, n_k_heads=0, q_in=None, k_out=None))


def test_rotate_refuses_what_is_not_a_gpu_tensor():
    x = torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16)
    for args in ((x, x), (None, None), (x, None), (7, 7), (x[0], x[0])):
        assert status(prompt.rotate, prompt.make_rope(128), *args, first=None) == pask.PASK_E_ARG


def attn_args(**kw):
    d = dict(cache=fake_cache(), layer=0, batch=2, max_q=70, n_q=None, first=None, q=AT, out=AT, lse=None,
             softmax_scale=0.1, max_ctx_hint=0, ws=AT, ws_bytes=1 << 40)
    d.update(kw)
    return d


@pytest.mark.parametrize("bad, want", [
    (dict(layer=-1), "SHAPE"), (dict(layer=2), "SHAPE"), (dict(batch=0), "SHAPE"), (dict(batch=5), "SHAPE"),
    (dict(max_q=-1), "SHAPE"), (dict(max_q=5001), "SHAPE"), (dict(q=None), "ARG"), (dict(out=None), "ARG"),
    (dict(q=AT + 8), "ARG"), (dict(out=AT + 2), "ARG"), (dict(lse=AT + 2), "ARG"), (dict(n_q=AT + 1), "ARG"),
    (dict(first=AT + 3), "ARG"), (dict(softmax_scale=math.nan), "ARG"), (dict(softmax_scale=math.inf), "ARG"),
    (dict(softmax_scale=3e38), "ARG"), (dict(ws=None), "ARG"), (dict(ws=AT + 128), "ARG"),
    (dict(ws_bytes=1000), "CAPACITY")])
def test_attention_refusals(bad, want):
    assert status(prompt.pask_prompt_attn, **attn_args(**bad)) == getattr(pask, "PASK_E_" + want)


def test_attention_refuses_a_broken_cache():
    assert status(prompt.pask_prompt_attn, **attn_args(cache=fake_cache(at=None))) == pask.PASK_E_ARG
    assert status(prompt.pask_prompt_attn, **attn_args(cache=fake_cache(at=AT + 64))) == pask.PASK_E_ARG
    c = fake_cache()
    c.bytes -= 1
    assert status(prompt.pask_prompt_attn, **attn_args(cache=c)) == pask.PASK_E_CAPACITY
    c = fake_cache()
    c.geom.head_dim = 96
    assert status(prompt.pask_prompt_attn, **attn_args(cache=c)) == pask.PASK_E_SHAPE
    big = geom(max_batch=60000, max_tokens_per_seq=1 << 20, n_q_heads=64, n_kv_heads=8)
    assert status(prompt.pask_prompt_attn, **attn_args(cache=fake_cache(big), batch=60000, max_q=1 << 20)) == pask.PASK_E_SHAPE


def test_attention_of_no_queries_is_ok():
    prompt.pask_prompt_attn(**attn_args(max_q=0, ws=None, ws_bytes=0))


def test_workspace_bytes():
    ws = lambda g, *a: prompt.pask_prompt_workspace_bytes(g, *a)
    g = geom(max_batch=64, max_tokens_per_seq=1 << 18)
    assert ws(g, 1, 1, 1 << 18) > 0                   # a long axis and few rows: cut
    assert ws(g, 1, 1, 16) == 0 or ws(g, 1, 1, 16) < ws(g, 1, 1, 1 << 18)
    assert ws(g, 64, 8192, 1 << 18) == 0              # enough tiles
    assert ws(g, 1, 4, 0) == ws(g, 1, 4, 1 << 18) == ws(g, 1, 4, (1 << 18) + 5)
    assert ws(g, 0, 4, 0) == ws(g, 65, 4, 0) == ws(g, 1, 0, 0) == ws(g, 1, -1, 0) == 0
    assert ws(geom(head_dim=96), 1, 4, 0) == 0


def test_workspace_of_any_call_is_bounded_and_asked_for():
    """At most 1,024 workgroups of 256 rows leave partial results; one byte less is refused."""
    import random
    rng = random.Random(5)
    for _ in range(400):
        group, kv, d = rng.choice([1, 2, 4, 8]), rng.randint(1, 8), rng.choice([64, 128])
        g = geom(max_batch=rng.randint(1, 300), n_q_heads=group * kv, n_kv_heads=kv, head_dim=d,
                 max_tokens_per_seq=1 << rng.randint(4, 17), recent_window=rng.choice([0, 5]))
        batch = rng.randint(1, g.max_batch)
        max_q = max(1, int(g.max_tokens_per_seq * rng.random() ** 4))
        need = prompt.pask_prompt_workspace_bytes(g, batch, max_q, 0)
        assert need <= 2048 * 256 * (d + 2) * 4 + 1024
        if need:
            assert need % 256 == 0
            args = attn_args(cache=fake_cache(g), batch=batch, max_q=max_q, ws_bytes=need - 1)
            assert status(prompt.pask_prompt_attn, **args) == pask.PASK_E_CAPACITY
