"""Python binding of the entry points of include/pask_prompt.h: rotary
positions and the attention of many query tokens over the mixed cache, one
function per entry point with the same name, on the statuses, caches and
pointer rules of the `pask` module.  make_rope() is pask_rope_init with
defaults; rotate() is pask_rope_apply for torch tensors, shapes and strides
taken from them.  The attention's tensors are checked by PaskSession.prompt.
"""

from __future__ import annotations

import ctypes as C

import torch

from . import pask
from .pask import PASK_E_ARG, PASK_E_SHAPE, PaskError, _check, _ptr

EXPORTS = ("pask_rope_init", "pask_rope_apply", "pask_prompt_workspace_bytes", "pask_prompt_attn")
PASK_ROPE_MAX_PAIRS, PASK_ROPE_MAX_HEAD_DIM, PASK_ROPE_MAX_HEADS = 128, 1024, 1024
PASK_ROPE_HALF, PASK_ROPE_INTERLEAVED = 0, 1
PASK_ROPE_PLAIN, PASK_ROPE_LINEAR, PASK_ROPE_BASE, PASK_ROPE_PARTS = 0, 1, 2, 3


class pask_rope(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("head_dim", "rot_first", "rot_dim", "layout")] + \
               [("magnitude", C.c_float), ("reserved", C.c_int32), ("turns", C.c_double * PASK_ROPE_MAX_PAIRS)]


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # not in torch's public interface
_lib = pask.library()
_P, _I, _L = C.c_void_p, C.c_int32, C.c_int64
_ROPE, _CACHE = C.POINTER(pask_rope), C.POINTER(pask.pask_cache)
_lib.pask_rope_init.argtypes = [_ROPE, _I, _I, _I, _I, C.c_double, _I, C.c_double, _I, C.c_double, C.c_double, C.c_float]
_lib.pask_rope_apply.argtypes = [_ROPE, _I, _I, _P, _P, _L, _P] + [_I, _P, _L, _P, _L] * 2 + [_P]
_lib.pask_prompt_workspace_bytes.restype = C.c_size_t
_lib.pask_prompt_workspace_bytes.argtypes = [C.POINTER(pask.pask_geom), _I, _I, _I]
_lib.pask_prompt_attn.argtypes = [_CACHE, _I, _I, _I, _P, _P, _P, _P, _P, C.c_float, _I, _P, C.c_size_t, _P]


def pask_rope_init(head_dim: int, rot_first: int, rot_dim: int, layout: int, base: float, scaling: int, factor: float,
                   original_len: int, low_turns: float, high_turns: float, magnitude: float) -> pask_rope:
    out = pask_rope()
    _check(_lib.pask_rope_init(C.byref(out), int(head_dim), int(rot_first), int(rot_dim), int(layout), float(base),
                               int(scaling), float(factor), int(original_len), float(low_turns), float(high_turns),
                               float(magnitude)), "pask_rope_init")
    return out


def make_rope(head_dim: int, base: float = 10000.0, *, rot_first: int = 0, rot_dim: int | None = None,
              layout: int = PASK_ROPE_HALF, scaling: int = PASK_ROPE_PLAIN, factor: float = 1.0, original_len: int = 1,
              low_turns: float = 1.0, high_turns: float = 32.0, magnitude: float = 1.0) -> pask_rope:
    """A rotation of heads of head_dim elements; all elements behind rot_first when rot_dim is None."""
    return pask_rope_init(head_dim, rot_first, head_dim - rot_first if rot_dim is None else rot_dim, layout, base,
                          scaling, factor, original_len, low_turns, high_turns, magnitude)


def pask_rope_apply(rope: pask_rope, batch: int, max_new: int, n_new, first, first_stride: int, pos, n_q_heads: int, q_in,
                    q_in_stride: int, q_out, q_out_stride: int, n_k_heads: int, k_in, k_in_stride: int, k_out,
                    k_out_stride: int, stream=0) -> None:
    _check(_lib.pask_rope_apply(C.byref(rope), int(batch), int(max_new), _ptr(n_new), _ptr(first), int(first_stride),
                                _ptr(pos), int(n_q_heads), _ptr(q_in), int(q_in_stride), _ptr(q_out), int(q_out_stride),
                                int(n_k_heads), _ptr(k_in), int(k_in_stride), _ptr(k_out), int(k_out_stride),
                                _ptr(stream)), "pask_rope_apply")


def pask_prompt_workspace_bytes(geom: pask.pask_geom, batch: int, max_q: int, max_ctx_hint: int) -> int:
    return int(_lib.pask_prompt_workspace_bytes(C.byref(geom), int(batch), int(max_q), int(max_ctx_hint)))


def pask_prompt_attn(cache: pask.pask_cache, layer: int, batch: int, max_q: int, n_q, first, q, out, lse=None,
                     softmax_scale: float = 1.0, max_ctx_hint: int = 0, ws=None, ws_bytes: int = 0, stream=0) -> None:
    _check(_lib.pask_prompt_attn(C.byref(cache), int(layer), int(batch), int(max_q), _ptr(n_q), _ptr(first), _ptr(q),
                                 _ptr(out), _ptr(lse), float(softmax_scale), int(max_ctx_hint), _ptr(ws), int(ws_bytes),
                                 _ptr(stream)), "pask_prompt_attn")


def _rows(name: str, t, shape, head_dim: int, device) -> int:
    """Elements between the rows of t, bf16 [batch, max_new, heads, head_dim] with contiguous heads and evenly spaced
    rows; PaskError if it is not that."""
    if not isinstance(t, torch.Tensor):
        raise PaskError(PASK_E_ARG, f"{name}: a tensor expected, got {type(t).__name__}")
    if t.dtype != torch.bfloat16 or t.device != device:
        raise PaskError(PASK_E_ARG, f"{name}: bfloat16 on {device} expected, got {t.dtype} on {t.device}")
    if t.dim() != 4 or t.shape[:2] != shape[:2] or t.shape[3] != head_dim:
        raise PaskError(PASK_E_SHAPE, f"{name}: shape ({shape[0]}, {shape[1]}, heads, {head_dim}) expected, got "
                                      f"{tuple(t.shape)}")
    batch, max_new, heads = t.shape[:3]
    if t.is_contiguous():
        return heads * head_dim
    s = t.stride()
    row = s[1] if max_new > 1 else s[0] if batch > 1 else heads * head_dim
    even = batch <= 1 or max_new <= 1 or s[0] == max_new * row
    if (head_dim > 1 and s[3] != 1) or (heads > 1 and s[2] != head_dim) or not even or row < heads * head_dim:
        raise PaskError(PASK_E_ARG, f"{name}: contiguous heads in evenly spaced rows expected, got strides {s}")
    return row


def rotate(rope: pask_rope, q, q_out, k=None, k_out=None, *, first=None, first_stride: int = 1, pos=None,
           n_new=None) -> None:
    """Rotate queries and keys on their device and its current stream.

    q, q_out, k, k_out bf16 [batch, max_new, heads, head_dim]; rows may lie apart (slices of a fused projection's
    rows), heads are contiguous; an output may be its input.  q and q_out, or k and k_out, may be None.  Token i of
    sequence b is at pos[b, i] (int32 [batch, max_new]), or at first[b * first_stride] + i (int32, e.g. [batch]).
    n_new int32 [batch]: the tokens of each sequence; rows behind them are left alone."""
    some = q if q is not None else k
    if not isinstance(some, torch.Tensor) or some.dim() != 4:
        raise PaskError(PASK_E_ARG, "rotate: q or k, tensors of four dimensions, expected")
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise PaskError(PASK_E_ARG, "rotate: an input without its output, or an output without its input")
    dev, shape = some.device, some.shape
    batch, max_new = shape[:2]
    if dev.type != "cuda":
        raise PaskError(PASK_E_ARG, "rotate: tensors on a GPU expected")
    sides = []
    for name, x, y in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            sides += [0, None, 0, None, 0]
            continue
        ins = _rows(name, x, shape, rope.head_dim, dev)
        outs = _rows(name + "_out", y, shape, rope.head_dim, dev)
        if x.shape != y.shape:
            raise PaskError(PASK_E_SHAPE, f"{name}_out: shape {tuple(x.shape)} expected, got {tuple(y.shape)}")
        sides += [x.shape[2], x, ins, y, outs]
    _ints("n_new", n_new, batch, dev)
    if pos is not None:
        _ints("pos", pos, batch * max_new, dev)
        if not pos.is_contiguous():
            raise PaskError(PASK_E_ARG, "pos: a contiguous tensor expected")
    if first is not None:
        if first_stride < 1:
            raise PaskError(PASK_E_ARG, "rotate: first_stride below 1")
        _ints("first", first, (batch - 1) * first_stride + 1 if batch else 0, dev, exact=False)
    if batch == 0 or max_new == 0:
        return
    args = (rope, batch, max_new, n_new, first, first_stride, pos, *sides)
    if torch.cuda.current_device() == dev.index:
        pask_rope_apply(*args, _stream(dev))
    else:
        with torch.cuda.device(dev):
            pask_rope_apply(*args, _stream(dev))


def _stream(device) -> int:
    """The raw handle of the device's current stream (torch's Stream object costs 2 us more, where that can be avoided)."""
    return _raw_stream(device.index) if _raw_stream else torch.cuda.current_stream(device).cuda_stream


def _ints(name: str, t, n: int, device, exact: bool = True) -> None:
    """Raises PaskError unless t is None or a contiguous int32 tensor of n (or, not exact, of n or more) elements."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.device != device or not t.is_contiguous():
        raise PaskError(PASK_E_ARG, f"{name}: a contiguous int32 tensor on {device} expected")
    if t.numel() != n if exact else t.numel() < n:
        raise PaskError(PASK_E_SHAPE, f"{name}: {n} elements expected, got {t.numel()}")
