"""What a layer over sampled neighbourhoods has around its attention: the residual's addition with the RMS norm, products in 8-bit integers for
serving, the gated pair of projections, and the clipping of gradients (argument checks and marshalling only; the kernels are the library's).

As in layer.py: arguments that make no sense raise LegionPrepError before anything is launched, results and workspaces are allocated for the stream that the
kernels run on, and a negative entry of pos (int32[tokens]) says that a row holds no token: whatever it holds, its results are zeros, and it counts for nothing.  add_norm and
gated_linear are differentiable, but for forward-mode derivatives, which are refused.  No derivative passes through rows in 8 bits, a norm of gradients or clipping.
"""
from __future__ import annotations

import struct

import torch
from torch.autograd.function import once_differentiable

from .binding import _Gated, _Residual, _Rows8, load_library
from .layer import _DTYPE, _ECAPACITY, _bad, _ints, _new, _no_tangents, _ok, _on, _packer, _ptr, _rows2, _workspace

_residual, _rows8, _gated = _packer(_Residual), _packer(_Rows8), _packer(_Gated)
_ACT = {"silu": 0, "gelu": 1}


def _plain(t, shape, name: str, dtype, index: int):
    """A tensor like this, rows end to end."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise _bad(f"{name}: {list(shape)}, {dtype}, on cuda:{index}")
    return t.contiguous()


def _vector(t, n: int, index: int, name: str):
    if t.dtype is not torch.float32 or t.get_device() != index or t.numel() != n or not t.is_contiguous():
        raise _bad(f"{name}: float32[{n}] on cuda:{index}")
    return t.data_ptr()


def _sum(x, residual, weight, pos, eps: float):
    """(device, arguments, type of the sum): x may be absent (backward)."""
    of = residual if x is None else x
    row, index, (tokens, width) = _rows2(of, "residual" if x is None else "x"), of.get_device(), of.shape
    if residual is None or residual is of:
        r_at, r_row, stream = (0, 0, of.dtype) if residual is None else (of.data_ptr(), row, of.dtype)
    else:
        r_row, r_at, stream = _rows2(residual, "residual"), residual.data_ptr(), residual.dtype
        if residual.shape != of.shape or residual.get_device() != index:
            raise _bad("residual: like x, where it is")
    if of.dtype not in _DTYPE or (stream is not of.dtype and stream is not torch.float32):
        raise _bad("x: float32, float16 or bfloat16; residual: of that type or float32")
    return index, (0 if x is None else x.data_ptr(), r_at, 0 if x is None else row, r_row, tokens, width), stream, (_vector(weight, width, index, "weight"),
                                                                                                                   _ints(pos, tokens, index, "pos"), eps)


def _residual_of(at, dtype, stream, rest):
    try:
        return _residual(*at, _DTYPE[dtype], _DTYPE[stream], *rest)
    except (OverflowError, struct.error):
        raise _bad("eps: a number that float32 holds") from None


class _AddNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, pos, eps):
        y, total = add_norm(x, residual, weight, pos, eps)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(total, weight, pos)
        ctx.of = x.dtype, residual is not None, eps
        return (y, total) if residual is not None else (y, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, d_total):
        total, weight, pos = ctx.saved_tensors
        dtype, adds, eps = ctx.of
        if dy is None:
            if d_total is None:
                return None, None, None, None, None
            dy = torch.zeros(total.shape, dtype=dtype, device=total.device)
        dx, d_residual, d_weight = add_norm_backward(dy, d_total, total, weight, pos, eps)
        return dx, d_residual if adds else None, d_weight, None, None


def add_norm(x, residual, weight, pos=None, eps: float = 1e-6, stream=None):
    """(y, total): total = x + residual, and its RMS norm y = total * weight / sqrt(mean(total^2) + eps).

    x [tokens, width] (float32, float16 or bfloat16, width up to 16384, values of a row side by side), residual like x, in the type of x or in float32, weight
    float32[width].  total has the type of the residual and y that of x; y is the norm of the total as it is rounded.  Without a residual (None) total is x
    itself."""
    _no_tangents(x, residual, weight)
    if (x.requires_grad or weight.requires_grad or (residual is not None and residual.requires_grad)) and torch.is_grad_enabled():
        with _on(x.get_device(), stream):
            y, total = _AddNorm.apply(x, residual, weight, pos, eps)
        return y, x if residual is None else total
    L = load_library()
    index, at, kind, rest = _sum(x, residual, weight, pos, eps)
    r = _residual_of(at, x.dtype, kind, rest)
    with _on(index, stream) as on:
        y, total = _new(x), x if residual is None else _new(residual)
        _ok(L.lgp_add_norm(index, r, y.data_ptr(), total.data_ptr(), on))
    return y, total


def add_norm_backward(dy, d_total, total, weight, pos=None, eps: float = 1e-6, stream=None):
    """Gradients (dx, d_residual, d_weight) of add_norm, from those of its results (d_total: None where nothing else uses the total), the total and the other
    arguments.  dx has the type of dy; where the total has the same, dx and d_residual are the same tensor."""
    L = load_library()
    dtype, kind = dy.dtype, total.dtype
    index, at, _, rest = _sum(None, total, weight, pos, eps)
    if dtype not in _DTYPE or (kind is not dtype and kind is not torch.float32):
        raise _bad("dy: float32, float16 or bfloat16; total: of that type or float32")
    r = _residual_of(at, dtype, kind, rest)
    with _on(index, stream) as on:
        dy = _plain(dy, total.shape, "dy", dtype, index)
        d_total = None if d_total is None else _plain(d_total, total.shape, "d_total", kind, index)
        d = _new(total)
        dx = d if kind is dtype else torch.empty(total.shape, dtype=dtype, device=total.device)
        dw = torch.empty_like(weight)
        w, size = _workspace(index, total.device, L.lgp_add_norm_workspace, r)
        _ok(L.lgp_add_norm_backward(index, r, dy.data_ptr(), _ptr(d_total), 0 if dx is d else dx.data_ptr(), d.data_ptr(), dw.data_ptr(), _ptr(w), size, on))
    return dx, d, dw


class Rows8:
    """Rows in 8-bit integers, -127 to 127: values (int8[tokens, width rounded up to 16], zeros behind width) times scales (float32[tokens]); of activations, or of the
    channels of a weight [out, width]."""

    def __init__(self, values, scales, width: int, pos=None):
        index = values.get_device()
        if (index < 0 or values.dim() != 2 or values.dtype is not torch.int8 or width < 1 or values.shape[1] != (width + 15) // 16 * 16 or
                not values.is_contiguous() or values.data_ptr() % 16):
            raise _bad("values: contiguous int8[tokens, width rounded up to 16], on a GPU, aligned to 16 bytes")
        tokens = values.shape[0]
        if scales.dtype is not torch.float32 or scales.get_device() != index or scales.shape != (tokens,) or not scales.is_contiguous():
            raise _bad("scales: contiguous float32[tokens]")
        self._set(values, scales, int(width), pos, index, _ints(pos, tokens, index, "pos"))

    def _set(self, values, scales, width, pos, index, pos_ptr):
        self.values, self.scales, self.width, self.pos, self.index = values, scales, width, pos, index
        self.c = _rows8(values.shape[0], width, values.data_ptr(), scales.data_ptr(), pos_ptr)
        return self

    @property
    def shape(self):
        return (self.values.shape[0], self.width)


def _new_rows8(tokens: int, width: int, pos, index: int, device, pos_ptr):
    values = torch.empty((tokens, (width + 15) // 16 * 16), dtype=torch.int8, device=device)
    return Rows8.__new__(Rows8)._set(values, torch.empty(tokens, dtype=torch.float32, device=device), width, pos, index, pos_ptr)


def pack_rows(x, pos=None, stream=None) -> Rows8:
    """x [tokens, width] (float32, float16 or bfloat16, width up to 16384, values of a row side by side) in 8 bits with a scale for each row, max |x| / 127;
    activations, or a weight [out, width]."""
    L = load_library()
    row, index, (tokens, width) = _rows2(x, "x"), x.get_device(), x.shape
    if x.dtype not in _DTYPE or width < 1:
        raise _bad("x: float32, float16 or bfloat16, one value in a row at least")
    pos_ptr = _ints(pos, tokens, index, "pos")
    with _on(index, stream) as on:
        rows = _new_rows8(tokens, width, pos, index, x.device, pos_ptr)
        _ok(L.lgp_pack_rows8(index, x.data_ptr(), row, _DTYPE[x.dtype], rows.c, on))
    return rows


def add_norm_rows8(x, residual, weight, pos=None, eps: float = 1e-6, stream=None):
    """(rows, total): add_norm with its result in 8 bits, as linear_rows8 takes it, from the 32-bit values of y.  No gradients pass."""
    L = load_library()
    index, at, kind, rest = _sum(x, residual, weight, pos, eps)
    r = _residual_of(at, x.dtype, kind, rest)
    with _on(index, stream) as on:
        rows = _new_rows8(*x.shape, pos, index, x.device, rest[1])
        total = x if residual is None else _new(residual)
        _ok(L.lgp_add_norm_rows8(index, r, rows.c, total.data_ptr(), on))
    return rows, total


def linear_rows8(rows: Rows8, weight: Rows8, bias=None, dtype=torch.bfloat16, stream=None):
    """rows weight^T + bias, [tokens, channels] in `dtype` (float32, float16 or bfloat16): a product of 8-bit integers, exact up to its scales.  weight: a Rows8 of
    [channels, width], as pack_rows gives it; bias: float32[channels].  No gradients pass."""
    L = load_library()
    index, channels = rows.index, weight.values.shape[0]
    if weight.index != index or weight.width != rows.width or weight.pos is not None or not channels:
        raise _bad(f"weight: rows of {rows.width} on cuda:{index}, one at least, all of them there")
    if dtype not in _DTYPE:
        raise _bad("dtype: float32, float16 or bfloat16")
    at = 0 if bias is None else _vector(bias, channels, index, "bias")
    with _on(index, stream) as on:
        out = torch.empty((rows.values.shape[0], channels), dtype=dtype, device=rows.values.device)
        _ok(L.lgp_linear_rows8(index, rows.c, weight.c, at, _DTYPE[dtype], out.data_ptr(), on))
    return out


def _pair(x, w_gate, w_up, act: str, pos):
    """(device, arguments) of the gated pair."""
    row, index, dtype, (tokens, width) = _rows2(x, "x"), x.get_device(), x.dtype, x.shape
    if dtype is not torch.float16 and dtype is not torch.bfloat16:
        raise _bad("x: float16 or bfloat16")
    for w, name in ((w_gate, "w_gate"), (w_up, "w_up")):
        if w.dtype is not dtype or w.get_device() != index or w.dim() != 2 or w.shape[1] != width or not w.is_contiguous() or w.data_ptr() % 16:
            raise _bad(f"{name}: [hidden, {width}], {dtype}, on cuda:{index}, rows end to end, aligned to 16 bytes")
    if w_gate.shape != w_up.shape:
        raise _bad("w_up: like w_gate")
    at = x.data_ptr()
    if tokens < 2:
        row = width
    if width % 8 or ((row % 8 or at % 16 or row >= 1 << 22) and tokens):
        raise _bad("x: a width and a stride between rows in multiples of 8, the stride below 2^22, aligned to 16 bytes")
    if act not in _ACT:
        raise _bad("act: silu or gelu")
    return index, _gated(at, row, tokens, width, w_gate.shape[0], _DTYPE[dtype], _ACT[act], w_gate.data_ptr(), w_up.data_ptr(), _ints(pos, tokens, index, "pos"))


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, act, pos):
        ctx.save_for_backward(x, w_gate, w_up, pos)
        ctx.act = act
        return gated_linear(x, w_gate, w_up, act, pos)

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        x, w_gate, w_up, pos = ctx.saved_tensors
        return *gated_linear_backward(dh, x, w_gate, w_up, ctx.act, pos), None, None


def gated_linear(x, w_gate, w_up, act: str = "silu", pos=None, stream=None):
    """act(x w_gate^T) * (x w_up^T), [tokens, hidden]: what stands before the last projection of a gated feed-forward block.

    x [tokens, width] and the weights [hidden, width]: float16 or bfloat16, width a multiple of 8.  act: "silu" or "gelu" (of the error function).  For its
    gradients nothing but x and the weights is kept."""
    _no_tangents(x, w_gate, w_up)
    if (x.requires_grad or w_gate.requires_grad or w_up.requires_grad) and torch.is_grad_enabled():
        with _on(x.get_device(), stream):
            return _GatedLinear.apply(x, w_gate, w_up, act, pos)
    L = load_library()
    index, g = _pair(x, w_gate, w_up, act, pos)
    with _on(index, stream) as on:
        h = torch.empty((x.shape[0], w_gate.shape[0]), dtype=x.dtype, device=x.device)
        st = L.lgp_gated_linear(index, g, h.data_ptr(), 0, 0, on)
        if st == _ECAPACITY:                    # nothing was launched: few calls want a workspace
            w, size = _workspace(index, x.device, L.lgp_gated_linear_workspace, g, 0)
            st = L.lgp_gated_linear(index, g, h.data_ptr(), _ptr(w), size, on)
        _ok(st)
    return h


def gated_linear_backward(dh, x, w_gate, w_up, act: str = "silu", pos=None, stream=None):
    """Gradients (dx, dw_gate, dw_up) of gated_linear, in the type of x, from that of its result; the other arguments are what it was given.

    Sums are in 32 bits.  The gradients of both projections' results are rounded to the type of x between the products (not for up to 8 tokens, or 64 with few hidden
    elements); float16's are lifted by a power of two for that, so that they may be beyond its range."""
    L = load_library()
    index, g = _pair(x, w_gate, w_up, act, pos)
    with _on(index, stream) as on:
        dh = _plain(dh, (x.shape[0], w_gate.shape[0]), "dh", x.dtype, index)
        dx = _new(x)
        dg, du = torch.empty_like(w_gate), torch.empty_like(w_up)
        w, size = _workspace(index, x.device, L.lgp_gated_linear_workspace, g, 1)
        _ok(L.lgp_gated_linear_backward(index, g, dh.data_ptr(), dx.data_ptr(), dg.data_ptr(), du.data_ptr(), _ptr(w), size, on))
    return dx, dg, du


def _clip(grads, most: float, out, stream):
    L = load_library()
    grads = [grads] if isinstance(grads, torch.Tensor) else list(grads)
    stays = out is None
    out = grads if stays else [out] if isinstance(out, torch.Tensor) else list(out)
    if not grads or len(out) != len(grads):
        raise _bad("grads: one tensor at least; out: as many")
    index, at = grads[0].get_device(), []
    for g, o in zip(grads, out):
        dtype = g.dtype
        if dtype not in _DTYPE or g.layout is not torch.strided or g.get_device() != index or index < 0 or not g.is_contiguous():
            raise _bad(f"grads: contiguous float32, float16 or bfloat16, all on one GPU, cuda:{index}")
        if o is not g and (o.dtype is not dtype or o.shape != g.shape or o.layout is not torch.strided or o.get_device() != index or not o.is_contiguous()):
            raise _bad("out: like grads, contiguous")
        at += (g.data_ptr(), o.data_ptr(), g.numel(), _DTYPE[dtype])
    try:
        code = struct.pack(f"@{len(at)}q", *at)
        most = float(most)
    except (OverflowError, TypeError, ValueError):
        raise _bad("most: a number") from None
    with _on(index, stream) as on:
        norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
        w, size = _workspace(index, norm.device, L.lgp_clip_gradients_workspace)
        _ok(L.lgp_clip_gradients(index, code, len(grads), most, norm.data_ptr(), _ptr(w), size, on))
    if most < float("inf") or not stays:
        torch.autograd.graph.increment_version(out)
    return norm


def gradient_norm(grads, stream=None) -> torch.Tensor:
    """The root of the sum of all squares (float32, no dimensions, on the GPU) over a tensor or many: contiguous float32, float16 and bfloat16 in any mixture."""
    return _clip(grads, float("inf"), None, stream)


def clip_gradients(grads, most: float, out=None, stream=None) -> torch.Tensor:
    """Scales gradients (as gradient_norm takes them) by min(1, most / norm) where they are, or into `out`, tensors like them; the norm before that.  Where the norm is
    not finite they are left, or copied, as they are.  No two of the tensors that are written may overlap."""
    return _clip(grads, most, out, stream)
