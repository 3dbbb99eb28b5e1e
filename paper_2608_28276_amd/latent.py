"""Python binding of the latent-attention entry points of libpask.so, declared
in include/pask_latent.h: one function per entry point with the same name, on
the statuses, policies and pointer rules of the `pask` module.  prompt_attn()
is pask_latent_prompt_attn, or pask_latent_prompt_attn_pos, for torch tensors,
shapes taken from them.
"""

from __future__ import annotations

import ctypes as C
import math

import torch

from . import pask
from .pask import _check, _ptr

EXPORTS = ("pask_latent_cache_layout_query", "pask_latent_cache_bytes", "pask_latent_cache_init",
           "pask_latent_cache_reset", "pask_latent_append", "pask_latent_read", "pask_latent_workspace_bytes",
           "pask_latent_decode_attn", "pask_latent_prompt_attn", "pask_latent_prompt_attn_pos",
           "pask_latent_cache_stats")
PASK_LATENT_MAX_HEADS = 128


class pask_latent_geom(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("max_batch", "n_layers", "n_q_heads", "rank", "rope_dim", "page_tokens",
                                         "max_tokens_per_seq", "hi_pages", "lo_pages")]


class pask_latent_cache(C.Structure):
    _fields_ = [("geom", pask_latent_geom), ("base", C.c_void_p), ("bytes", C.c_uint64)]


_lib = pask.library()
_P, _I = C.c_void_p, C.c_int32
_G, _CACHE, _POL = C.POINTER(pask_latent_geom), C.POINTER(pask_latent_cache), C.POINTER(pask.pask_policy)
_lib.pask_latent_cache_layout_query.argtypes = [_G, C.POINTER(pask.pask_cache_layout)]
_lib.pask_latent_cache_bytes.restype = C.c_size_t
_lib.pask_latent_cache_bytes.argtypes = [_G]
_lib.pask_latent_cache_init.argtypes = [_CACHE, _G, _P, C.c_size_t, _P]
_lib.pask_latent_cache_reset.argtypes = [_CACHE, _P]
_lib.pask_latent_append.argtypes = [_POL, _CACHE, _I, _I, _P, _I, _P, _P, _P, C.c_uint32, _P]
_lib.pask_latent_read.argtypes = [_CACHE, _I, _I, _I, _P, _P, _P, _P, _P]
_lib.pask_latent_workspace_bytes.restype = C.c_size_t
_lib.pask_latent_workspace_bytes.argtypes = [_G, _I, _I]
_lib.pask_latent_decode_attn.argtypes = [_POL, _CACHE, _I, _I, _P, _P, _P, _P, _P, _P, C.c_float, _I, _P, C.c_size_t,
                                         _P]
_lib.pask_latent_prompt_attn.argtypes = [_I] * 8 + [_P] * 7 + [C.c_float, _P]
_lib.pask_latent_prompt_attn_pos.argtypes = [_I] * 8 + [_P] * 9 + [C.c_float, _P]
_lib.pask_latent_cache_stats.argtypes = [_POL, _CACHE, _I, C.POINTER(pask.pask_stats), _P]


def make_latent_geom(**kw) -> pask_latent_geom:
    g = pask_latent_geom()
    g.page_tokens = 16
    for k, v in kw.items():
        setattr(g, k, int(v))
    return g


def pask_latent_cache_layout_query(geom: pask_latent_geom) -> pask.pask_cache_layout:
    out = pask.pask_cache_layout()
    _check(_lib.pask_latent_cache_layout_query(C.byref(geom), C.byref(out)), "pask_latent_cache_layout_query")
    return out


def pask_latent_cache_bytes(geom: pask_latent_geom) -> int:
    return int(_lib.pask_latent_cache_bytes(C.byref(geom)))


def pask_latent_cache_init(cache: pask_latent_cache, geom: pask_latent_geom, base, nbytes: int, stream=0) -> None:
    _check(_lib.pask_latent_cache_init(C.byref(cache), C.byref(geom), _ptr(base), int(nbytes), _ptr(stream)),
           "pask_latent_cache_init")


def pask_latent_cache_reset(cache: pask_latent_cache, stream=0) -> None:
    _check(_lib.pask_latent_cache_reset(C.byref(cache), _ptr(stream)), "pask_latent_cache_reset")


def pask_latent_append(policy, cache: pask_latent_cache, layer: int, batch: int, n_new, max_new: int, tags, c, r,
                       flags: int = 0, stream=0) -> None:
    _check(_lib.pask_latent_append(C.byref(policy), C.byref(cache), int(layer), int(batch), _ptr(n_new), int(max_new),
                                   _ptr(tags), _ptr(c), _ptr(r), int(flags), _ptr(stream)), "pask_latent_append")


def pask_latent_read(cache: pask_latent_cache, layer: int, batch: int, rows: int, c, r, pos, cu, stream=0) -> None:
    _check(_lib.pask_latent_read(C.byref(cache), int(layer), int(batch), int(rows), _ptr(c), _ptr(r), _ptr(pos),
                                 _ptr(cu), _ptr(stream)), "pask_latent_read")


def pask_latent_workspace_bytes(geom: pask_latent_geom, batch: int, max_ctx_hint: int) -> int:
    return int(_lib.pask_latent_workspace_bytes(C.byref(geom), int(batch), int(max_ctx_hint)))


def pask_latent_decode_attn(policy, cache: pask_latent_cache, layer: int, batch: int, q, out, lse=None, tags_new=None,
                            c_new=None, r_new=None, softmax_scale: float = 1.0, max_ctx_hint: int = 0, ws=None,
                            ws_bytes: int = 0, stream=0) -> None:
    _check(_lib.pask_latent_decode_attn(C.byref(policy), C.byref(cache), int(layer), int(batch), _ptr(q), _ptr(out),
                                        _ptr(lse), _ptr(tags_new), _ptr(c_new), _ptr(r_new), float(softmax_scale),
                                        int(max_ctx_hint), _ptr(ws), int(ws_bytes), _ptr(stream)),
           "pask_latent_decode_attn")


def pask_latent_prompt_attn(batch: int, n_heads: int, nope_dim: int, rope_dim: int, v_dim: int, max_q: int,
                            total_q: int, total_k: int, cu_q, cu_k, q, kv, r, out, lse=None,
                            softmax_scale: float = 1.0, stream=0) -> None:
    _check(_lib.pask_latent_prompt_attn(int(batch), int(n_heads), int(nope_dim), int(rope_dim), int(v_dim), int(max_q),
                                        int(total_q), int(total_k), _ptr(cu_q), _ptr(cu_k), _ptr(q), _ptr(kv), _ptr(r),
                                        _ptr(out), _ptr(lse), float(softmax_scale), _ptr(stream)),
           "pask_latent_prompt_attn")


def pask_latent_prompt_attn_pos(batch: int, n_heads: int, nope_dim: int, rope_dim: int, v_dim: int, max_q: int,
                                total_q: int, total_k: int, cu_q, cu_k, pos, q_first, q, kv, r, out, lse=None,
                                softmax_scale: float = 1.0, stream=0) -> None:
    _check(_lib.pask_latent_prompt_attn_pos(int(batch), int(n_heads), int(nope_dim), int(rope_dim), int(v_dim),
                                            int(max_q), int(total_q), int(total_k), _ptr(cu_q), _ptr(cu_k), _ptr(pos),
                                            _ptr(q_first), _ptr(q), _ptr(kv), _ptr(r), _ptr(out), _ptr(lse),
                                            float(softmax_scale), _ptr(stream)),
           "pask_latent_prompt_attn_pos")


def pask_latent_cache_stats(policy, cache: pask_latent_cache, batch: int, stream=0):
    """Returns (stats, status); status is PASK_OK or PASK_E_DEVICE_FLAG."""
    out = pask.pask_stats()
    st = _lib.pask_latent_cache_stats(C.byref(policy), C.byref(cache), int(batch), C.byref(out), _ptr(stream))
    if st not in (pask.PASK_OK, pask.PASK_E_DEVICE_FLAG):
        raise pask.PaskError(st, "pask_latent_cache_stats")
    return out, st


def check_tensor(name: str, t, dtype, shape, device) -> None:
    """Raises PaskError unless t is a contiguous tensor of this type, shape and device (a None in shape fits any size)."""
    if not isinstance(t, torch.Tensor):
        raise pask.PaskError(pask.PASK_E_ARG, f"{name}: a tensor expected, got {type(t).__name__}")
    if t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise pask.PaskError(pask.PASK_E_ARG, f"{name}: contiguous {dtype} on {device} expected, got {t.dtype} "
                                              f"{'' if t.is_contiguous() else 'strided '}on {t.device}")
    if len(t.shape) != len(shape) or any(w is not None and w != g for w, g in zip(shape, t.shape)):
        raise pask.PaskError(pask.PASK_E_SHAPE, f"{name}: shape {tuple(shape)} expected, got {tuple(t.shape)}")


def prompt_attn(q, kv, r, out, lse, cu_q, cu_k, max_q: int, softmax_scale: float | None = None, pos=None,
                q_first=None) -> None:
    """Causal attention of packed prompts in the expanded form, on q's device and its current stream.

    q bf16 [total_q, heads, nope + rope], kv bf16 [total_k, heads, nope + v], r bf16 [total_k, rope], out bf16
    [total_q, heads, v], lse fp32 [total_q, heads] or None, cu_q and cu_k int32 [batch + 1].  Sequence b's queries are
    the last of its keys; or, with pos int32 [total_k] (the keys' positions, as the cache's read-back returns them) and
    q_first int32 [batch] (the position of each sequence's first query), query i sees the keys at q_first[b] + i and
    before.  softmax_scale: 1 / sqrt(nope + rope) when None."""
    for name, t in (("q", q), ("kv", kv), ("r", r), ("out", out), ("cu_q", cu_q), ("cu_k", cu_k)):
        if not isinstance(t, torch.Tensor):
            raise pask.PaskError(pask.PASK_E_ARG, f"{name}: a tensor expected, got {type(t).__name__}")
    dev = q.device
    if dev.type != "cuda":
        raise pask.PaskError(pask.PASK_E_ARG, "prompt_attn: tensors on a GPU expected")
    if q.dim() != 3 or kv.dim() != 3 or r.dim() != 2 or out.dim() != 3 or cu_q.dim() != 1:
        raise pask.PaskError(pask.PASK_E_SHAPE, "prompt_attn: q, kv, out of three, r of two, cu_q of one dimension expected")
    total_q, heads, qk = q.shape
    rope, v = r.shape[1], out.shape[2]
    nope, batch = qk - rope, cu_q.shape[0] - 1
    bf16 = torch.bfloat16
    check_tensor("q", q, bf16, (total_q, heads, qk), dev)
    check_tensor("kv", kv, bf16, (None, heads, nope + v), dev)
    check_tensor("r", r, bf16, (kv.shape[0], rope), dev)
    check_tensor("out", out, bf16, (total_q, heads, v), dev)
    check_tensor("cu_q", cu_q, torch.int32, (batch + 1,), dev)
    check_tensor("cu_k", cu_k, torch.int32, (batch + 1,), dev)
    if lse is not None:
        check_tensor("lse", lse, torch.float32, (total_q, heads), dev)
    sizes = (batch, heads, nope, rope, v, max_q, total_q, kv.shape[0])
    scale = 1.0 / math.sqrt(qk) if softmax_scale is None else softmax_scale
    if pos is None and q_first is None:
        with torch.cuda.device(dev):
            pask_latent_prompt_attn(*sizes, cu_q, cu_k, q, kv, r, out, lse, scale,
                                    torch.cuda.current_stream(dev).cuda_stream)
        return
    check_tensor("pos", pos, torch.int32, (kv.shape[0],), dev)
    check_tensor("q_first", q_first, torch.int32, (batch,), dev)
    with torch.cuda.device(dev):
        pask_latent_prompt_attn_pos(*sizes, cu_q, cu_k, pos, q_first, q, kv, r, out, lse, scale,
                                    torch.cuda.current_stream(dev).cuda_stream)
