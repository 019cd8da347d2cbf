"""Binding of the workers' local-gradient operators (include/lossy_local.h):
embedding lookup and gradient, 8-bit activation checkpoints and the weight
gradient that reads them.

Argument marshalling only, like the rest of the package: device pointers,
sizes and the current stream of the tensors' device go to the C entry point of
the same name; a non-zero return code is raised.  Activations are
[n][t][width] tensors (any row stride, workers `t` rows apart), grads and
replicas the [n][ld] row buffers of the lossy step.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import LL_BF16, LL_F32, _SIGNATURES, _check, _f32, _i32, _i64, _load, _need_numel, _vp

__all__ = ["ll_embed", "ll_embed_grad", "ll_embed_grad_workspace_bytes", "ll_act_pack",
           "ll_act_unpack", "ll_act_wgrad", "ll_act_wgrad_workspace_bytes",
           "LL_ACT_GROUP", "LL_I32", "LL_I64"]

LL_I32, LL_I64 = 0, 1
LL_ACT_GROUP = 32

_sz = ctypes.c_size_t
_SIGNATURES.update({
    "ll_embed": (ctypes.c_int, [_i32, _i64, _i64, _i64, _i64, _i32, _vp, _i64, _vp, _i32, _vp,
                                _i64, _i64, _f32, _i32, _vp, _i64, _vp]),
    "ll_embed_grad": (ctypes.c_int, [_i32, _i64, _i64, _i64, _i64, _i32, _vp, _i64, _vp, _i32,
                                     _vp, _i64, _f32, _i32, _vp, _i64, _i64, _i32, _vp, _sz,
                                     _vp]),
    "ll_embed_grad_workspace_bytes": (_sz, [_i32, _i64, _i64, _i64]),
    "ll_act_pack": (ctypes.c_int, [_i32, _i64, _i64, _vp, _i32, _vp, _i64, _vp, _i64, _vp, _i64,
                                   _vp]),
    "ll_act_unpack": (ctypes.c_int, [_i32, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _i32, _vp,
                                     _i64, _vp]),
    "ll_act_wgrad": (ctypes.c_int, [_i32, _i64, _i64, _i64, _vp, _i32, _vp, _i64, _vp, _i64, _vp,
                                    _i64, _f32, _i32, _vp, _i64, _i64, _i32, _vp, _sz, _vp]),
    "ll_act_wgrad_workspace_bytes": (_sz, [_i32, _i64, _i64, _i64]),
})

# Called with GPU tensors in hand only; a torch without GPU support, where the
# package can be imported all the same, has neither.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)

_FLOATS = {torch.float32: LL_F32, torch.bfloat16: LL_BF16}
_INTS = {torch.int32: LL_I32, torch.int64: LL_I64}


def _on_device(name: str, first: torch.Tensor, *others) -> int:
    """Index of the one GPU that all tensors of a call are on."""
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            dev = -1
    if dev < 0:
        raise ValueError(f"{name} needs all its tensors on one GPU, got "
                         f"{sorted({str(t.device) for t in (first, *others) if t is not None})}")
    return dev


def _call(name: str, dev: int, *args) -> None:
    """The C entry point on the tensors' device and its current stream (the
    handle alone: a small call is bound by the host)."""
    fn = getattr(_load(), name)
    if _current_device() == dev:
        code = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            code = fn(*args, _raw_stream(dev))
    if code:
        _check(name, code)


def _code(t: torch.Tensor, name: str, codes: dict) -> int:
    code = codes.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be one of {[str(d) for d in codes]}, got {t.dtype}")
    return code


def _act(t: torch.Tensor, name: str, n: int, tokens: int, width: Optional[int] = None) -> int:
    """Row stride of an [n][tokens][width] tensor whose workers lie `tokens`
    rows apart."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[0] != n or shape[1] != tokens:
        raise ValueError(f"{name} must be [{n}][{tokens}][...], got {tuple(shape)}")
    if width is not None and shape[2] != width:
        raise ValueError(f"{name} must have width {width}, got {shape[2]}")
    if stride[2] != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have unit column stride")
    # the stride of a dimension of length 1 means nothing
    ld = stride[1] if tokens > 1 else (stride[0] if n > 1 else shape[2])
    if n > 1 and tokens > 0 and stride[0] != tokens * ld:
        raise ValueError(f"{name}: workers must lie {tokens} rows apart, got strides {stride}")
    return ld


def _tokens(t: torch.Tensor) -> tuple:
    """(n, tokens, ld, integer code) of the token ids."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2:
        raise ValueError(f"tokens must be 2-D, got {tuple(shape)}")
    n, m = shape
    if stride[1] != 1 and m > 1:
        raise ValueError("tokens must have unit column stride")
    return n, m, (stride[0] if n > 1 else max(m, 1)), _code(t, "tokens", _INTS)


def _row_buffer(t: torch.Tensor, name: str, n: int, offset: int, rows: int, h: int) -> tuple:
    """(ld, dtype code) of an [n][ld] row buffer that holds rows x h elements
    at `offset`."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[0] != n:
        raise ValueError(f"{name} must be [{n}][ld], got {tuple(shape)}")
    width = shape[1]
    if stride[1] != 1 and width > 1:
        raise ValueError(f"{name} must have unit column stride")
    if offset < 0 or offset + rows * h > width:
        raise ValueError(f"{name}: {rows} rows of {h} elements at offset {offset} exceed its "
                         f"{width} columns")
    # one row: its stride counts where it is one, else its length
    ld = stride[0] if n > 1 else max(stride[0], width)
    return ld, _code(t, name, _FLOATS)


def _lens(t: Optional[torch.Tensor], n: int):
    if t is None:
        return None
    _need_numel(t, "lengths", n, torch.int32)
    if not t.is_contiguous():
        raise ValueError("lengths must be contiguous")
    return t.data_ptr()


def _ws(t: Optional[torch.Tensor]) -> tuple:
    if t is None:
        return None, 0
    if not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _codes(q: torch.Tensor, s: torch.Tensor, n: int, tokens: int, h: int) -> tuple:
    """(ld_q, ld_s) of an 8-bit checkpoint."""
    for t, name in ((q, "q"), (s, "s")):
        if t.dtype != torch.uint8:
            raise ValueError(f"{name} must be uint8, got {t.dtype}")
    return (_act(q, "q", n, tokens, h),
            _act(s, "s", n, tokens, (h + LL_ACT_GROUP - 1) // LL_ACT_GROUP))


def ll_embed(tokens: torch.Tensor, replicas: torch.Tensor, out: torch.Tensor, *, v: int,
             first: int = 0, offset: int = 0, scale: float = 1.0,
             lengths: Optional[torch.Tensor] = None) -> None:
    """out[i][j] = scale * row (tokens[i][j] - first) of the v-row table at
    element `offset` of replicas[i]; zeros for tokens outside the table."""
    n, m, ld_t, it = _tokens(tokens)
    ld_o = _act(out, "out", n, m)
    h = out.shape[2]
    ld_r, rt = _row_buffer(replicas, "replicas", n, offset, v, h)
    ot, lens = _code(out, "out", _FLOATS), _lens(lengths, n)
    dev = _on_device("ll_embed", tokens, replicas, out, lengths)
    _call("ll_embed", dev, n, m, h, v, first, it, tokens.data_ptr(), ld_t, lens, rt,
          replicas.data_ptr(), ld_r, offset, scale, ot, out.data_ptr(), ld_o)


def ll_embed_grad_workspace_bytes(n: int, t: int, h: int, v: int) -> int:
    return int(_load().ll_embed_grad_workspace_bytes(n, t, h, v))


def ll_embed_grad(tokens: torch.Tensor, dy: torch.Tensor, grads: torch.Tensor, *, v: int,
                  first: int = 0, offset: int = 0, scale: float = 1.0, accumulate: bool = False,
                  lengths: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> None:
    """Gradient of ll_embed: scale times the sum of dy over each table row's
    tokens, into (accumulate: added to) the table at `offset` of grads."""
    n, m, ld_t, it = _tokens(tokens)
    ld_y = _act(dy, "dy", n, m)
    h = dy.shape[2]
    ld_g, gt = _row_buffer(grads, "grads", n, offset, v, h)
    yt, lens = _code(dy, "dy", _FLOATS), _lens(lengths, n)
    ws, ws_bytes = _ws(workspace)
    dev = _on_device("ll_embed_grad", tokens, dy, grads, lengths, workspace)
    _call("ll_embed_grad", dev, n, m, h, v, first, it, tokens.data_ptr(), ld_t, lens, yt,
          dy.data_ptr(), ld_y, scale, gt, grads.data_ptr(), ld_g, offset, int(accumulate), ws,
          ws_bytes)


def ll_act_pack(x: torch.Tensor, q: torch.Tensor, s: torch.Tensor, *,
                lengths: Optional[torch.Tensor] = None) -> None:
    """8-bit checkpoint of x [n][t][h]: e4m3 codes q [n][t][h] and exponent
    bytes s [n][t][ceil(h / 32)], both uint8."""
    if x.dim() != 3:
        raise ValueError(f"x must be 3-D, got {tuple(x.shape)}")
    n, m, h = x.shape
    ld_x = _act(x, "x", n, m)
    ld_q, ld_s = _codes(q, s, n, m, h)
    xt, lens = _code(x, "x", _FLOATS), _lens(lengths, n)
    dev = _on_device("ll_act_pack", x, q, s, lengths)
    _call("ll_act_pack", dev, n, m, h, lens, xt, x.data_ptr(), ld_x, q.data_ptr(), ld_q,
          s.data_ptr(), ld_s)


def ll_act_unpack(q: torch.Tensor, s: torch.Tensor, out: torch.Tensor, *,
                  lengths: Optional[torch.Tensor] = None) -> None:
    """The activations of an 8-bit checkpoint, exact in out's dtype."""
    if out.dim() != 3:
        raise ValueError(f"out must be 3-D, got {tuple(out.shape)}")
    n, m, h = out.shape
    ld_o = _act(out, "out", n, m)
    ld_q, ld_s = _codes(q, s, n, m, h)
    ot, lens = _code(out, "out", _FLOATS), _lens(lengths, n)
    dev = _on_device("ll_act_unpack", q, s, out, lengths)
    _call("ll_act_unpack", dev, n, m, h, lens, q.data_ptr(), ld_q, s.data_ptr(), ld_s, ot,
          out.data_ptr(), ld_o)


def ll_act_wgrad_workspace_bytes(n: int, t: int, o: int, h: int) -> int:
    return int(_load().ll_act_wgrad_workspace_bytes(n, t, o, h))


def ll_act_wgrad(dy: torch.Tensor, q: torch.Tensor, s: torch.Tensor, grads: torch.Tensor, *,
                 offset: int = 0, scale: float = 1.0, accumulate: bool = False,
                 lengths: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> None:
    """Weight gradient scale * dy^T x of a linear layer whose input x is kept
    as the checkpoint (q, s): [o][h] at `offset` of every row of grads."""
    if dy.dim() != 3 or q.dim() != 3:
        raise ValueError(f"dy and q must be 3-D, got {tuple(dy.shape)} and {tuple(q.shape)}")
    n, m, o = dy.shape
    h = q.shape[2]
    ld_y = _act(dy, "dy", n, m)
    ld_q, ld_s = _codes(q, s, n, m, h)
    ld_g, gt = _row_buffer(grads, "grads", n, offset, o, h)
    yt, lens = _code(dy, "dy", _FLOATS), _lens(lengths, n)
    ws, ws_bytes = _ws(workspace)
    dev = _on_device("ll_act_wgrad", dy, q, s, grads, lengths, workspace)
    _call("ll_act_wgrad", dev, n, m, o, h, lens, yt, dy.data_ptr(), ld_y, q.data_ptr(), ld_q,
          s.data_ptr(), ld_s, scale, gt, grads.data_ptr(), ld_g, offset, int(accumulate), ws,
          ws_bytes)
