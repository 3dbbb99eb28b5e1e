"""The latent-attention entry points on the host (no GPU): exports, geometry
and layout, and every refusal, none of which may reach a HIP call."""

import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from workload.policy import make_policy, pack_blob

from . import latent_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pask = pytest.importorskip("paper_2608_28276_amd.pask", reason="libpask.so not built")
latent = pytest.importorskip("paper_2608_28276_amd.latent")


def geom(**kw):
    d = dict(max_batch=4, n_layers=2, n_q_heads=20, rank=512, rope_dim=64, max_tokens_per_seq=500, hi_pages=40,
             lo_pages=30)
    d.update(kw)
    return latent.make_latent_geom(**d)


def policy(layers=2, window=0):
    pol = make_policy(6, 2, layers, 0.33, 1)
    pol.recent_window = window
    return pask.pask_policy_load(pack_blob(pol), None)


def fake_cache(g=None, at=256 * 1024):
    """A cache whose buffer is an address that nothing may touch."""
    c = latent.pask_latent_cache()
    c.geom = g or geom()
    c.base = at
    c.bytes = latent.pask_latent_cache_bytes(c.geom)
    return c


def status(f, *args, **kw):
    with pytest.raises(pask.PaskError) as e:
        f(*args, **kw)
    return e.value.status


def test_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "pask_latent.h")).read()
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(pask_\w+)\s*\(", text, re.M))
    assert names == set(latent.EXPORTS)
    for n in names:
        assert hasattr(pask.library(), n) and hasattr(latent, n), n


@pytest.mark.parametrize("rank, rope", [(128, 32), (128, 64), (256, 32), (256, 64), (512, 32), (512, 64)])
def test_layout(rank, rope):
    g = geom(rank=rank, rope_dim=rope)
    L = latent.pask_latent_cache_layout_query(g)
    assert L.hi_page_bytes == 16 * 2 * (rank + rope)
    assert L.lo_page_bytes == 16 * (rank // 2 + rank // 16 + 2 * rope)
    assert (L.max_pages, L.counter_stride, L.ring_pages) == (32, 8, 0)
    offs = [L.status_off, L.counters_off, L.block_table_off, L.index_list_off, L.staging_off, L.budget_off,
            L.hi_pool_off, L.lo_pool_off, L.total_bytes]
    assert offs == sorted(offs) and L.status_off == 0
    assert L.index_list_off - L.block_table_off >= 4 * 2 * 2 * 4 * 32
    assert L.lo_pool_off - L.hi_pool_off >= 40 * L.hi_page_bytes
    assert L.total_bytes - L.lo_pool_off >= 30 * L.lo_page_bytes
    assert latent.pask_latent_cache_bytes(g) == L.total_bytes


@pytest.mark.parametrize("bad", [dict(max_batch=0), dict(max_batch=65536), dict(n_layers=0), dict(n_layers=129),
                                 dict(n_q_heads=0), dict(n_q_heads=129), dict(rank=64), dict(rank=384), dict(rank=0),
                                 dict(rope_dim=0), dict(rope_dim=48), dict(rope_dim=128), dict(page_tokens=32),
                                 dict(max_tokens_per_seq=0), dict(max_tokens_per_seq=(1 << 28) + 1),
                                 dict(hi_pages=-1), dict(lo_pages=-1)])
def test_unsupported_geometry(bad):
    g = geom(**bad)
    assert latent.pask_latent_cache_bytes(g) == 0
    assert latent.pask_latent_workspace_bytes(g, 1, 100) == 0
    assert status(latent.pask_latent_cache_layout_query, g) == pask.PASK_E_SHAPE
    c = latent.pask_latent_cache()
    assert status(latent.pask_latent_cache_init, c, g, 4096, 1 << 40) == pask.PASK_E_SHAPE
    c = fake_cache()
    c.geom = g
    assert status(latent.pask_latent_cache_reset, c) == pask.PASK_E_SHAPE


def test_workspace():
    g = geom()
    w = latent.pask_latent_workspace_bytes(g, 4, 500)
    assert w > 0 and w % 256 == 0
    assert latent.pask_latent_workspace_bytes(g, 4, 0) == w == latent.pask_latent_workspace_bytes(g, 4, 10 ** 6)
    assert latent.pask_latent_workspace_bytes(g, 1, 100) <= w
    assert latent.pask_latent_workspace_bytes(g, 0, 100) == 0 == latent.pask_latent_workspace_bytes(g, 5, 100)


def test_cache_refusals():
    g, c = geom(), latent.pask_latent_cache()
    n = latent.pask_latent_cache_bytes(g)
    init = latent.pask_latent_cache_init
    assert status(init, c, g, 0, n) == pask.PASK_E_ARG
    assert status(init, c, g, 4096 + 128, n) == pask.PASK_E_ARG
    assert status(init, c, g, 4096, n - 1) == pask.PASK_E_CAPACITY
    bad = fake_cache()
    bad.base = None
    assert status(latent.pask_latent_cache_reset, bad) == pask.PASK_E_ARG
    bad = fake_cache(at=64)
    assert status(latent.pask_latent_cache_reset, bad) == pask.PASK_E_ARG
    bad = fake_cache()
    bad.bytes -= 1
    assert status(latent.pask_latent_cache_reset, bad) == pask.PASK_E_CAPACITY


A = 1 << 20                                          # stands for an aligned device address


@pytest.mark.parametrize("want, over", [
    ("PASK_E_SHAPE", dict(layer=2)), ("PASK_E_SHAPE", dict(layer=-1)), ("PASK_E_SHAPE", dict(batch=0)),
    ("PASK_E_SHAPE", dict(batch=5)), ("PASK_E_SHAPE", dict(max_new=-1)), ("PASK_E_SHAPE", dict(max_new=501)),
    ("PASK_E_ARG", dict(flags=2)), ("PASK_E_ARG", dict(c=0)), ("PASK_E_ARG", dict(r=0)), ("PASK_E_ARG", dict(c=A + 8)),
    ("PASK_E_ARG", dict(r=A + 2)), ("PASK_E_ARG", dict(tags=0)), ("PASK_E_ARG", dict(n_new=A + 2))])
def test_append_refusals(want, over):
    a = dict(layer=0, batch=2, n_new=0, max_new=3, tags=A, c=A, r=A, flags=0)
    a.update(over)
    assert status(latent.pask_latent_append, policy(), fake_cache(), **a) == getattr(pask, want)


def test_append_of_nothing_is_no_call():
    latent.pask_latent_append(policy(), fake_cache(), 0, 2, 0, 0, A, A, A)


def test_policy_refusals():
    args = (0, 2, 0, 3, A, A, A)
    assert status(latent.pask_latent_append, policy(window=8), fake_cache(), *args) == pask.PASK_E_UNSUPPORTED
    assert status(latent.pask_latent_append, policy(layers=4), fake_cache(), *args) == pask.PASK_E_SHAPE
    bad = policy()
    bad.n_tags = 0
    assert status(latent.pask_latent_append, bad, fake_cache(), *args) == pask.PASK_E_POLICY
    bad = policy()
    bad.group_of_layer[1] = 9
    assert status(latent.pask_latent_append, bad, fake_cache(), *args) == pask.PASK_E_POLICY


@pytest.mark.parametrize("want, over", [
    ("PASK_E_SHAPE", dict(layer=2)), ("PASK_E_SHAPE", dict(batch=0)), ("PASK_E_SHAPE", dict(batch=5)),
    ("PASK_E_ARG", dict(rows=-1)), ("PASK_E_ARG", dict(c=0)), ("PASK_E_ARG", dict(c=A + 8)), ("PASK_E_ARG", dict(r=0)),
    ("PASK_E_ARG", dict(r=A + 4)), ("PASK_E_ARG", dict(pos=A + 1)), ("PASK_E_ARG", dict(cu=0)),
    ("PASK_E_ARG", dict(cu=A + 2))])
def test_read_refusals(want, over):
    a = dict(layer=0, batch=2, rows=10, c=A, r=A, pos=A, cu=A)
    a.update(over)
    assert status(latent.pask_latent_read, fake_cache(), **a) == getattr(pask, want)


def test_read_of_more_rows_than_offsets_hold():
    c = fake_cache(geom(max_batch=65535, max_tokens_per_seq=40000))
    assert status(latent.pask_latent_read, c, 0, 65535, 10, A, A, A, A) == pask.PASK_E_SHAPE


@pytest.mark.parametrize("want, over", [
    ("PASK_E_SHAPE", dict(layer=-1)), ("PASK_E_SHAPE", dict(batch=5)), ("PASK_E_ARG", dict(q=0)),
    ("PASK_E_ARG", dict(q=A + 8)), ("PASK_E_ARG", dict(out=0)), ("PASK_E_ARG", dict(out=A + 2)),
    ("PASK_E_ARG", dict(lse=A + 2)), ("PASK_E_ARG", dict(tags_new=A, c_new=0, r_new=A)),
    ("PASK_E_ARG", dict(tags_new=A, c_new=A, r_new=A + 8)), ("PASK_E_ARG", dict(softmax_scale=float("nan"))),
    ("PASK_E_ARG", dict(softmax_scale=float("inf"))), ("PASK_E_ARG", dict(ws=0)), ("PASK_E_ARG", dict(ws=A + 128)),
    ("PASK_E_CAPACITY", dict(ws_bytes=1000))])
def test_decode_refusals(want, over):
    a = dict(layer=0, batch=2, q=A, out=A, ws=A, ws_bytes=1 << 40)
    a.update(over)
    assert status(latent.pask_latent_decode_attn, policy(), fake_cache(), **a) == getattr(pask, want)


def test_decode_workspace_is_what_is_asked():
    c = fake_cache()
    n = latent.pask_latent_workspace_bytes(c.geom, 3, 200)
    a = dict(layer=0, batch=3, q=A, out=A, max_ctx_hint=200, ws=A, ws_bytes=n - 1)
    assert status(latent.pask_latent_decode_attn, policy(), c, **a) == pask.PASK_E_CAPACITY


PROMPT = dict(batch=2, n_heads=8, nope_dim=128, rope_dim=64, v_dim=128, max_q=10, total_q=20, total_k=30, cu_q=A, cu_k=A,
              q=A, kv=A, r=A, out=A)


@pytest.mark.parametrize("want, over", [
    ("PASK_E_SHAPE", dict(batch=0)), ("PASK_E_SHAPE", dict(batch=65536)), ("PASK_E_SHAPE", dict(n_heads=0)),
    ("PASK_E_SHAPE", dict(n_heads=129)), ("PASK_E_SHAPE", dict(nope_dim=96)), ("PASK_E_SHAPE", dict(v_dim=32)),
    ("PASK_E_SHAPE", dict(rope_dim=0)), ("PASK_E_ARG", dict(max_q=-1)), ("PASK_E_ARG", dict(total_q=-1)),
    ("PASK_E_ARG", dict(total_k=-1)), ("PASK_E_ARG", dict(cu_q=0)), ("PASK_E_ARG", dict(cu_k=A + 2)),
    ("PASK_E_ARG", dict(q=0)), ("PASK_E_ARG", dict(q=A + 8)), ("PASK_E_ARG", dict(kv=0)), ("PASK_E_ARG", dict(r=A + 2)),
    ("PASK_E_ARG", dict(out=0)), ("PASK_E_ARG", dict(lse=A + 1)), ("PASK_E_ARG", dict(softmax_scale=float("nan"))),
    ("PASK_E_SHAPE", dict(batch=65535, n_heads=128, max_q=1000, total_q=1 << 30))])
def test_prompt_refusals(want, over):
    a = dict(PROMPT)
    a.update(over)
    assert status(latent.pask_latent_prompt_attn, **a) == getattr(pask, want)


@pytest.mark.parametrize("over", [dict(max_q=0), dict(total_q=0, q=0, out=0)])
def test_prompt_of_no_query_is_no_call(over):
    latent.pask_latent_prompt_attn(**dict(PROMPT, **over))


def test_stats_refusals():
    out = pask.pask_stats()
    lib, c, p = pask.library(), fake_cache(), policy()
    assert lib.pask_latent_cache_stats(C.byref(p), C.byref(c), 5, C.byref(out), None) == pask.PASK_E_SHAPE
    assert lib.pask_latent_cache_stats(C.byref(p), C.byref(c), 2, None, None) == pask.PASK_E_ARG


def test_tensor_checks():
    t = torch.zeros(4, 6, dtype=torch.bfloat16)
    dev = t.device
    latent.check_tensor("t", t, torch.bfloat16, (4, None), dev)
    for bad, st in ((t.float(), pask.PASK_E_ARG), (t.t(), pask.PASK_E_ARG), (None, pask.PASK_E_ARG),
                    (t[:3], pask.PASK_E_SHAPE), (t[None], pask.PASK_E_SHAPE)):
        assert status(latent.check_tensor, "t", bad, torch.bfloat16, (4, 6), dev) == st
    assert status(latent.prompt_attn, t, t, t, t, None, t, t, 1) == pask.PASK_E_ARG        # not on a GPU


def test_reference_low_values():
    """The reference's own format, on values worked out by hand."""
    x = np.zeros((1, 64))
    x[0, :5] = [7.0, -3.5, 0.5, 1.5, 2.5]             # s = 1: ties go to even
    x[0, 32:34] = [2.0 ** 127, -1.0]                     # s saturates at 65504
    v = latent_ref.low_values(latent_ref.to_bf16(x))
    assert v[0, :5].tolist() == [7.0, -4.0, 0.0, 2.0, 2.0]
    assert v[0, 32] == latent_ref.to_bf16(np.array([7 * 65504.0]))[0] and v[0, 33] == 0.0
    tiny = np.full((1, 32), 2.0 ** -27)               # absmax / 7 rounds to an fp16 zero
    assert (latent_ref.low_values(tiny) == 0).all()


def test_the_recorded_attention_traffic_still_holds():
    """The counters in profiles/ are tied to the code of the attention kernels, which the latent ones leave alone."""
    import bench
    assert bench.traffic_record("qwen3_4b_b64_p1k-8k_g1024") is not None
