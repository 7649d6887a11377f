"""Operators of a model layer over sampled neighbourhoods: attention inside documents, norms of heads with rotation, and activations
held in 8 bits (argument checks and marshalling only; the kernels are the library's).

Arguments that make no sense raise LegionPrepError before anything is launched.  Results and workspaces are allocated for the stream
that the kernels run on.  attend and norm_rotate are differentiable: where a gradient is wanted of an input, their results carry it; forward-mode
derivatives are refused.  Packed activations are what a backward pass keeps, and no gradient passes through them.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from .binding import LegionPrepError, _Attention, _Documents, _Heads, _Packed, _raw_stream, load_library

_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_EINVAL, _ECAPACITY = -1, -3
_LARGE = 1 << 24              # strides from here on are looked at more closely


def _packer(structure):
    """struct.pack for a ctypes structure."""
    code = {C.c_void_p: "P", C.c_int64: "q", C.c_int32: "i", C.c_float: "f"}
    form = struct.Struct("@" + "".join(code[kind] for _, kind in structure._fields_) + "0P")
    assert form.size == C.sizeof(structure)
    return form.pack


_documents, _attention_of, _heads, _packed = (_packer(x) for x in (_Documents, _Attention, _Heads, _Packed))


def _bad(text: str) -> LegionPrepError:
    return LegionPrepError(_EINVAL, text)


def _ok(st: int):
    if st != 0:
        raise LegionPrepError(st, load_library().lgp_strerror(st).decode())


def _no_tangents(*tensors):
    """Forward-mode derivatives need no requires_grad and would be lost without a word."""
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise _bad("forward-mode derivatives are not computed")


class _Here:
    """The current stream, where results are allocated as they are."""
    __slots__ = ("ptr",)

    def __init__(self, index: int):
        self.ptr = torch.cuda.current_stream(index).cuda_stream if _raw_stream is None else _raw_stream(index)

    def __enter__(self):
        return self.ptr

    def __exit__(self, *exc):
        pass


class _There:
    """Another stream, which results are allocated for."""
    __slots__ = ("stream", "context")

    def __init__(self, stream):
        self.stream, self.context = stream, torch.cuda.stream(stream)

    def __enter__(self):
        self.context.__enter__()
        return self.stream.cuda_stream

    def __exit__(self, *exc):
        self.context.__exit__(*exc)


def _on(index: int, stream):
    if stream is None:
        return _Here(index)
    if stream.device_index != index:
        raise _bad(f"stream: of cuda:{index}, where the arguments are")
    return _There(stream)


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _ints(t, n: int, index: int, name: str):
    """The address of an optional int32 vector of n entries."""
    if t is None:
        return 0
    if t.dtype is not torch.int32 or t.get_device() != index or t.numel() != n or not t.is_contiguous():
        raise _bad(f"{name}: {n} contiguous int32 entries on cuda:{index}")
    return t.data_ptr()


def _heads_of(t, name: str, dtype, index: int):
    """The address and the strides of a [rows, heads, dim] tensor whose heads can be read 16 bytes at a time."""
    if t.dim() != 3 or t.dtype is not dtype or t.get_device() != index:
        raise _bad(f"{name}: [rows, heads, dim], {dtype}, on cuda:{index}")
    row, head, one = t.stride()
    at = t.data_ptr()
    if one != 1 or row % 8 or head % 8 or at % 16 or row >= _LARGE or head >= _LARGE:
        rows, heads, _ = t.shape
        row, head = row if rows > 1 else 0, head if heads > 1 else 0          # the stride of a single row or head says nothing
        if t.numel() and (one != 1 or row % 8 or head % 8 or at % 16):
            raise _bad(f"{name}: elements of a head side by side, strides in multiples of 8, aligned to 16 bytes")
        if not t.numel():
            row = head = 0
    return at, row, head


def _like(t, shape, name: str, dtype, index: int):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise _bad(f"{name}: {list(shape)}, {dtype}, on cuda:{index}")
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _new(t):
    """A tensor like t, rows end to end."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


class Documents:
    """Which rows of queries and of keys belong together.  Document d owns rows offsets[d] .. offsets[d + 1] (int32[n + 1], the first 0, the last
    the number of rows); the first lens[d] of them hold tokens (None: all).  q_pos and k_pos (int32, by row) are needed where scores fall
    with the distance.  The sampler's list of hop h is Documents(arange(n + 1), arange(n + 1) * fanout, k_lens=cnt[h])."""

    def __init__(self, q_offsets, k_offsets, q_lens=None, k_lens=None, q_pos=None, k_pos=None):
        n = q_offsets.numel() - 1
        index = q_offsets.get_device()
        if n < 0 or index < 0:
            raise _bad("q_offsets: one entry at least, on a GPU")
        self.index, self.q_pos, self.k_pos = index, q_pos, k_pos
        self._keep = (q_offsets, k_offsets, q_lens, k_lens)
        self._n = n
        self._at = (_ints(q_offsets, n + 1, index, "q_offsets"), _ints(k_offsets, n + 1, index, "k_offsets"), _ints(q_lens, n, index, "q_lens"),
                    _ints(k_lens, n, index, "k_lens"))

    def _rows(self, q_rows: int, k_rows: int) -> bytes:
        return _documents(self._n, q_rows, k_rows, *self._at, _ints(self.q_pos, q_rows, self.index, "q_pos"), _ints(self.k_pos, k_rows, self.index, "k_pos"))


def _attention(q, k, v, docs: Documents, slopes, cap: float, scale):
    index, dtype = docs.index, q.dtype
    if dtype is not torch.float16 and dtype is not torch.bfloat16:
        raise _bad("q, k and v: float16 or bfloat16")
    (qp, q_row, q_head), (kp, k_row, k_head), (vp, v_row, v_head) = _heads_of(q, "q", dtype, index), _heads_of(k, "k", dtype, index), _heads_of(v, "v", dtype, index)
    (q_rows, heads, dim), (k_rows, kv_heads, k_dim) = q.shape, k.shape
    if k.shape != v.shape or k_dim != dim or not kv_heads or not heads or heads % kv_heads:
        raise _bad("k and v: [rows, kv_heads, dim] with a kv_heads that divides the heads of q")
    if slopes is not None:
        if slopes.dtype is not torch.float32 or slopes.get_device() != index or slopes.numel() != heads or not slopes.is_contiguous():
            raise _bad("slopes: float32[heads]")
        if (docs.q_pos is None and q_rows) or (docs.k_pos is None and k_rows):
            raise _bad("slopes need positions of queries and keys")
    rows = docs._rows(q_rows, k_rows)
    try:
        return rows, _attention_of(qp, kp, vp, q_row, q_head, k_row, k_head, v_row, v_head, heads, kv_heads, dim, _DTYPE[dtype],
                                   dim ** -0.5 if scale is None else scale, cap, _ptr(slopes))
    except (OverflowError, struct.error):
        raise _bad("scale and cap: numbers that float32 holds") from None


def _workspace(index: int, device, query, *args):
    size = C.c_size_t()
    _ok(query(index, *args, C.byref(size)))
    return (torch.empty(size.value, dtype=torch.uint8, device=device) if size.value else None), size.value


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, slopes, docs, cap, scale):
        out, lse, rest = attend(q, k, v, docs, slopes=slopes, cap=cap, scale=scale, rest=True)
        ctx.save_for_backward(q, k, v, slopes, out, lse, rest)
        ctx.mark_non_differentiable(lse, rest)
        ctx.of = docs, cap, scale
        return out, lse, rest

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out, *_):
        q, k, v, slopes, out, lse, rest = ctx.saved_tensors
        docs, cap, scale = ctx.of
        return *attend_backward(d_out, q, k, v, out, lse, docs, rest=rest, slopes=slopes, cap=cap, scale=scale), None, None, None


def attend(q, k, v, docs: Documents, slopes=None, cap: float = 0.0, scale: float | None = None, rest: bool = False, stream=None):
    """Attention of every query to the keys of its document; (out, lse, rest).

    q [q_rows, heads, dim], k and v [k_rows, kv_heads, dim]: float16 or bfloat16, dim a multiple of 8 up to 128.  Scores are scale * q.k
    (dim^-1/2 by default), capped as cap * tanh(. / cap) where cap > 0, less slopes[head] * |q_pos - k_pos| where slopes (float32[heads]) are
    given.  out is like q, end to end; lse (float32[q_rows, heads]) is the logarithm of the sum of exp(score).  Queries without keys and rows
    without tokens get zeros and -inf.  rest: also return what the rounding of out took off, for attend_backward.  Gradients pass through out, not
    through lse or rest."""
    _no_tangents(q, k, v, slopes)
    if (q.requires_grad or k.requires_grad or v.requires_grad or (slopes is not None and slopes.requires_grad)) and torch.is_grad_enabled():
        with _on(docs.index, stream):
            out, lse, left = _Attend.apply(q, k, v, slopes, docs, cap, scale)
        return out, lse, left if rest else None
    L = load_library()
    d, a = _attention(q, k, v, docs, slopes, cap, scale)
    device = q.device
    with _on(docs.index, stream) as on:
        out = _new(q)
        left = _new(q) if rest else None
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=device)
        st = L.lgp_attend(docs.index, d, a, out.data_ptr(), _ptr(left), lse.data_ptr(), 0, 0, on)
        if st == _ECAPACITY:                    # nothing was launched: few calls want a workspace
            w, size = _workspace(docs.index, device, L.lgp_attend_workspace, d, a, 0)
            st = L.lgp_attend(docs.index, d, a, out.data_ptr(), _ptr(left), lse.data_ptr(), _ptr(w), size, on)
        _ok(st)
    return out, lse, left


def attend_backward(d_out, q, k, v, out, lse, docs: Documents, rest=None, slopes=None, cap: float = 0.0, scale: float | None = None, stream=None):
    """Gradients (dq, dk, dv, d_slopes) of attend by its inputs, from that of out and from what attend returned; d_slopes is None without slopes."""
    L = load_library()
    d, a = _attention(q, k, v, docs, slopes, cap, scale)
    index, dev = docs.index, q.device
    with _on(index, stream) as on:
        d_out, out = _like(d_out, q.shape, "d_out", q.dtype, index), _like(out, q.shape, "out", q.dtype, index)
        rest = None if rest is None else _like(rest, q.shape, "rest", q.dtype, index)
        lse = _like(lse, q.shape[:2], "lse", torch.float32, index)
        dq, dk, dv = _new(q), _new(k), _new(v)
        d_slopes = None if slopes is None else torch.empty_like(slopes)
        w, size = _workspace(index, dev, L.lgp_attend_workspace, d, a, 1)
        _ok(L.lgp_attend_backward(index, d, a, d_out.data_ptr(), out.data_ptr(), _ptr(rest), lse.data_ptr(), dq.data_ptr(),
                                  dk.data_ptr(), dv.data_ptr(), _ptr(d_slopes), _ptr(w), size, on))
    return dq, dk, dv, d_slopes


def rotation_table(positions: int, rot: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """float32[positions, rot]: cosines, then sines, of position * base^(-2 i / rot), computed in 64 bits."""
    if positions < 1 or rot < 1 or rot % 16:
        raise _bad("positions: one at least; rot: a multiple of 16")
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


def _weight(w, name: str, dim: int, index: int):
    at = w.data_ptr()
    if w.dtype is not torch.float32 or w.get_device() != index or w.numel() != dim or not w.is_contiguous() or at % 16:
        raise _bad(f"{name}: float32[dim], aligned to 16 bytes")
    return at


def _norm(q, k, q_weight, k_weight, pos, table, eps: float):
    index, dtype = q.get_device(), q.dtype
    if dtype not in _DTYPE or index < 0:
        raise _bad("q and k: float32, float16 or bfloat16, on a GPU")
    (qp, q_row, q_head), (kp, k_row, k_head) = _heads_of(q, "q", dtype, index), _heads_of(k, "k", dtype, index)
    (tokens, heads, dim), (k_tokens, kv_heads, k_dim) = q.shape, k.shape
    if k_tokens != tokens or k_dim != dim:
        raise _bad("k: [tokens, kv_heads, dim], as many tokens and elements as q")
    rot = n_pos = 0
    at = 0
    if table is not None:
        at = table.data_ptr()
        if table.dim() != 2 or table.dtype is not torch.float32 or table.get_device() != index or not table.is_contiguous() or at % 16 or pos is None:
            raise _bad("table: float32[positions, rot], aligned to 16 bytes, and pos with it")
        n_pos, rot = table.shape
    wq, wk, positions = _weight(q_weight, "q_weight", dim, index), _weight(k_weight, "k_weight", dim, index), _ints(pos, tokens, index, "pos")
    try:
        return index, _heads(qp, kp, q_row, q_head, k_row, k_head, tokens, heads, kv_heads, dim, _DTYPE[dtype], wq, wk, positions, rot, n_pos, at, eps)
    except (OverflowError, struct.error):
        raise _bad("eps: a number that float32 holds") from None


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, pos, table, eps):
        ctx.save_for_backward(q, k, q_weight, k_weight, pos, table)
        ctx.eps = eps
        return norm_rotate(q, k, q_weight, k_weight, pos, table, eps)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        return *norm_rotate_backward(dq_out, dk_out, *ctx.saved_tensors, eps=ctx.eps), None, None, None


def norm_rotate(q, k, q_weight, k_weight, pos=None, table=None, eps: float = 1e-6, stream=None):
    """RMS norm of every head of q [tokens, heads, dim] and k [tokens, kv_heads, dim] with weights (float32[dim]), and the rotation of its first
    table.shape[1] elements by the token's position (rotation_table); new tensors (q, k), rows end to end.  dim: a multiple of 8 up to 256.
    Rows of a negative pos have no token and become zeros; those of a position beyond the table become NaN."""
    _no_tangents(q, k, q_weight, k_weight)
    if (q.requires_grad or k.requires_grad or q_weight.requires_grad or k_weight.requires_grad) and torch.is_grad_enabled():
        with _on(q.get_device(), stream):
            return _NormRotate.apply(q, k, q_weight, k_weight, pos, table, eps)
    L = load_library()
    index, h = _norm(q, k, q_weight, k_weight, pos, table, eps)
    with _on(index, stream) as on:
        q_out, k_out = _new(q), _new(k)
        _ok(L.lgp_norm_rotate(index, h, q_out.data_ptr(), k_out.data_ptr(), on))
    return q_out, k_out


def norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, pos=None, table=None, eps: float = 1e-6, stream=None):
    """Gradients (dq, dk, dq_weight, dk_weight) of norm_rotate, from those of its results; the other arguments are what it was given."""
    L = load_library()
    index, h = _norm(q, k, q_weight, k_weight, pos, table, eps)
    dev = q.device
    with _on(index, stream) as on:
        dq_out, dk_out = _like(dq_out, q.shape, "dq_out", q.dtype, index), _like(dk_out, k.shape, "dk_out", k.dtype, index)
        dq, dk = _new(q), _new(k)
        dqw, dkw = torch.empty_like(q_weight), torch.empty_like(k_weight)
        w, size = _workspace(index, dev, L.lgp_norm_rotate_workspace, h)
        _ok(L.lgp_norm_rotate_backward(index, h, dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(), dk.data_ptr(), dqw.data_ptr(),
                                       dkw.data_ptr(), _ptr(w), size, on))
    return dq, dk, dqw, dkw


class PackedActivations:
    """Activations in 8 bits: values (int8[tokens, width rounded up to 16]) times 2^(exps - 127) (uint8[tokens, groups of 32])."""

    def __init__(self, values, exps, width: int, dtype, pos=None):
        index = values.get_device()
        if (index < 0 or values.dim() != 2 or values.dtype is not torch.int8 or width < 1 or values.shape[1] != (width + 15) // 16 * 16 or
                not values.is_contiguous() or values.data_ptr() % 16):
            raise _bad("values: contiguous int8[tokens, width rounded up to 16], on a GPU, aligned to 16 bytes")
        if exps.dtype is not torch.uint8 or exps.get_device() != index or exps.shape != (values.shape[0], (width + 31) // 32) or not exps.is_contiguous():
            raise _bad("exps: contiguous uint8[tokens, (width + 31) / 32]")
        if dtype not in _DTYPE:
            raise _bad("dtype: float32, float16 or bfloat16")
        self._set(values, exps, int(width), dtype, pos, index, _ints(pos, values.shape[0], index, "pos"))

    def _set(self, values, exps, width, dtype, pos, index, pos_ptr):
        self.values, self.exps, self.width, self.dtype, self.pos, self.index = values, exps, width, dtype, pos, index
        self.c = _packed(values.shape[0], width, _DTYPE[dtype], values.data_ptr(), exps.data_ptr(), pos_ptr)
        return self

    @property
    def shape(self):
        return (self.values.shape[0], self.width)


def _rows2(t, name: str):
    row, one = t.stride() if t.dim() == 2 else (0, 0)
    if t.get_device() < 0 or t.dim() != 2 or (one != 1 and t.shape[1] != 1 and t.numel()):
        raise _bad(f"{name}: [tokens, width] on a GPU, values of a row side by side")
    return row


def pack_activations(x, pos=None, stream=None) -> PackedActivations:
    """x [tokens, width] (float32, float16 or bfloat16, values of a row side by side) in 8 bits: 32 values of a row share a power of two.  Rows of a
    negative pos (int32[tokens]) hold no token: they are not read and packed as zeros."""
    L = load_library()
    row, index, dtype, device = _rows2(x, "x"), x.get_device(), x.dtype, x.device
    tokens, width = x.shape
    if dtype not in _DTYPE or width < 1:
        raise _bad("x: float32, float16 or bfloat16, one value in a row at least")
    pos_ptr = _ints(pos, tokens, index, "pos")
    with _on(index, stream) as on:
        values = torch.empty((tokens, (width + 15) // 16 * 16), dtype=torch.int8, device=device)
        exps = torch.empty((tokens, (width + 31) // 32), dtype=torch.uint8, device=device)
        packed = PackedActivations.__new__(PackedActivations)._set(values, exps, width, dtype, pos, index, pos_ptr)
        _ok(L.lgp_pack_activations(index, x.data_ptr(), row, packed.c, on))
    return packed


def unpack_activations(packed: PackedActivations, stream=None) -> torch.Tensor:
    """The values that `packed` stands for, in the type that came."""
    L = load_library()
    with _on(packed.index, stream) as on:
        x = torch.empty(packed.shape, dtype=packed.dtype, device=packed.values.device)
        _ok(L.lgp_unpack_activations(packed.index, packed.c, x.data_ptr(), on))
    return x


def packed_weight_grad(packed: PackedActivations, dy, bias: bool = True, stream=None):
    """(dw, db) of a linear layer y = x W^T + b whose input was packed: float32[out, width] and float32[out] (None if bias is False), from dy [tokens,
    out] in bfloat16, or in float16 if x was."""
    L = load_library()
    row, index, device = _rows2(dy, "dy"), packed.index, dy.device
    tokens, out = dy.shape
    if tokens != packed.values.shape[0] or out < 1 or dy.get_device() != index:
        raise _bad("dy: [tokens, out], where the packed rows are")
    if dy.dtype is not torch.bfloat16 and (dy.dtype is not torch.float16 or packed.dtype is not torch.float16):
        raise _bad("dy: bfloat16, or float16 with activations that came in float16")
    with _on(index, stream) as on:
        dw = torch.empty((out, packed.width), dtype=torch.float32, device=device)
        db = torch.empty(out, dtype=torch.float32, device=device) if bias else None
        w, size = _workspace(index, device, L.lgp_packed_weight_grad_workspace, packed.c, out)
        _ok(L.lgp_packed_weight_grad(index, packed.c, dy.data_ptr(), row, _DTYPE[dy.dtype], out, dw.data_ptr(), _ptr(db), _ptr(w), size, on))
    return dw, db
