"""Operators of a model layer over sampled neighbourhoods: attention inside documents, norms of heads with rotation, and activations
held in 8 bits (argument checks and marshalling only; the kernels are the library's).

Arguments that make no sense raise LegionPrepError before anything is launched.  Results and workspaces are allocated for the stream
that the kernels run on.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import LegionPrepError, _Attention, _Documents, _Heads, _Packed, _raw_stream, load_library

_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_EINVAL = -1


def _want(ok, text: str):
    if not ok:
        raise LegionPrepError(_EINVAL, text)


def _ok(st: int):
    if st != 0:
        raise LegionPrepError(st, load_library().lgp_strerror(st).decode())


class _On:
    """The stream a call runs on, which is also the one that its results are allocated for."""

    def __init__(self, device: torch.device, stream):
        self.index = device.index
        self.other = None
        if stream is not None:
            self.ptr = stream.cuda_stream
            self.other = torch.cuda.stream(stream)
        elif _raw_stream is not None:
            self.ptr = _raw_stream(self.index)
        else:
            self.ptr = torch.cuda.current_stream(device).cuda_stream

    def __enter__(self):
        if self.other is not None:
            self.other.__enter__()
        return self

    def __exit__(self, *exc):
        if self.other is not None:
            self.other.__exit__(*exc)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ints(t, n: int, device, name: str):
    """An optional int32 vector of n entries."""
    if t is not None:
        _want(t.dtype == torch.int32 and t.is_cuda and t.device == device and t.is_contiguous() and t.numel() == n,
              f"{name}: {n} contiguous int32 entries on {device}")


def _heads_of(t, name: str, dtype, device):
    """A [rows, heads, dim] tensor whose heads can be read 16 bytes at a time; its strides."""
    _want(t.dim() == 3 and t.dtype == dtype and t.device == device, f"{name}: [rows, heads, dim], {dtype}, on {device}")
    row, head, one = t.stride()
    if t.numel():
        _want(one == 1 and row % 8 == 0 and head % 8 == 0 and t.data_ptr() % 16 == 0,
              f"{name}: elements of a head side by side, strides in multiples of 8, aligned to 16 bytes")
    return row, head


def _like(t, shape, name: str, dtype, device):
    _want(tuple(t.shape) == tuple(shape) and t.dtype == dtype and t.device == device, f"{name}: {list(shape)}, {dtype}, on {device}")
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class Documents:
    """Which rows of queries and of keys belong together.  Document d owns rows offsets[d] .. offsets[d + 1] (int32[n + 1], the first 0, the last
    the number of rows); the first lens[d] of them hold tokens (None: all).  q_pos and k_pos (int32, by row) are needed where scores fall
    with the distance.  The sampler's list of hop h is Documents(arange(n + 1), arange(n + 1) * fanout, k_lens=cnt[h])."""

    def __init__(self, q_offsets, k_offsets, q_lens=None, k_lens=None, q_pos=None, k_pos=None):
        n = q_offsets.numel() - 1
        dev = q_offsets.device
        _want(n >= 0 and dev.type == "cuda", "q_offsets: one entry at least, on a GPU")
        _ints(q_offsets, n + 1, dev, "q_offsets")
        _ints(k_offsets, n + 1, dev, "k_offsets")
        _ints(q_lens, n, dev, "q_lens")
        _ints(k_lens, n, dev, "k_lens")
        self.device, self.q_pos, self.k_pos = dev, q_pos, k_pos
        self._keep = (q_offsets, k_offsets, q_lens, k_lens)
        self.c = _Documents(n, 0, 0, q_offsets.data_ptr(), k_offsets.data_ptr(), _ptr(q_lens), _ptr(k_lens), _ptr(q_pos), _ptr(k_pos))

    def _rows(self, q_rows: int, k_rows: int):
        _ints(self.q_pos, q_rows, self.device, "q_pos")
        _ints(self.k_pos, k_rows, self.device, "k_pos")
        self.c.q_rows, self.c.k_rows = q_rows, k_rows
        return self.c


def _attention(q, k, v, docs: Documents, slopes, cap: float, scale):
    dev = docs.device
    strides = _heads_of(q, "q", q.dtype, dev) + _heads_of(k, "k", q.dtype, dev) + _heads_of(v, "v", q.dtype, dev)
    heads, dim = q.shape[1:]
    _want(k.shape == v.shape and k.shape[2] == dim and k.shape[1] > 0 and heads > 0 and heads % k.shape[1] == 0,
          "k and v: [rows, kv_heads, dim] with a kv_heads that divides the heads of q")
    _want(q.dtype in (torch.float16, torch.bfloat16), "q, k and v: float16 or bfloat16")
    if slopes is not None:
        _want(slopes.dtype == torch.float32 and slopes.device == dev and slopes.is_contiguous() and slopes.numel() == heads, "slopes: float32[heads]")
        _want((docs.q_pos is not None or not q.shape[0]) and (docs.k_pos is not None or not k.shape[0]), "slopes need positions of queries and keys")
    return docs._rows(q.shape[0], k.shape[0]), _Attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), *strides, heads, k.shape[1], dim, _DTYPE[q.dtype],
                                                          dim ** -0.5 if scale is None else scale, cap, _ptr(slopes))


def _workspace(on: _On, device, query, *args):
    size = C.c_size_t()
    _ok(query(on.index, *args, C.byref(size)))
    return (torch.empty(size.value, dtype=torch.uint8, device=device) if size.value else None), size.value


def attend(q, k, v, docs: Documents, slopes=None, cap: float = 0.0, scale: float | None = None, rest: bool = False, stream=None):
    """Attention of every query to the keys of its document; (out, lse, rest).

    q [q_rows, heads, dim], k and v [k_rows, kv_heads, dim]: float16 or bfloat16, dim a multiple of 8 up to 128.  Scores are scale * q.k
    (dim^-1/2 by default), capped as cap * tanh(. / cap) where cap > 0, less slopes[head] * |q_pos - k_pos| where slopes (float32[heads]) are
    given.  out is like q, end to end; lse (float32[q_rows, heads]) is the logarithm of the sum of exp(score).  Queries without keys and rows
    without tokens get zeros and -inf.  rest: also return what the rounding of out took off, for attend_backward."""
    L = load_library()
    d, a = _attention(q, k, v, docs, slopes, cap, scale)
    with _On(docs.device, stream) as on:
        out = torch.empty(q.shape, dtype=q.dtype, device=docs.device)
        left = torch.empty_like(out) if rest else None
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=docs.device)
        w, size = _workspace(on, docs.device, L.lgp_attend_workspace, C.byref(d), C.byref(a), 0)
        _ok(L.lgp_attend(on.index, C.byref(d), C.byref(a), out.data_ptr(), _ptr(left), lse.data_ptr(), _ptr(w), size, on.ptr))
    return out, lse, left


def attend_backward(d_out, q, k, v, out, lse, docs: Documents, rest=None, slopes=None, cap: float = 0.0, scale: float | None = None, stream=None):
    """Gradients (dq, dk, dv, d_slopes) of attend by its inputs, from that of out and from what attend returned; d_slopes is None without slopes."""
    L = load_library()
    d, a = _attention(q, k, v, docs, slopes, cap, scale)
    dev = docs.device
    with _On(dev, stream) as on:
        d_out, out = _like(d_out, q.shape, "d_out", q.dtype, dev), _like(out, q.shape, "out", q.dtype, dev)
        rest = None if rest is None else _like(rest, q.shape, "rest", q.dtype, dev)
        lse = _like(lse, q.shape[:2], "lse", torch.float32, dev)
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
        d_slopes = None if slopes is None else torch.empty_like(slopes)
        w, size = _workspace(on, dev, L.lgp_attend_workspace, C.byref(d), C.byref(a), 1)
        _ok(L.lgp_attend_backward(on.index, C.byref(d), C.byref(a), d_out.data_ptr(), out.data_ptr(), _ptr(rest), lse.data_ptr(), dq.data_ptr(),
                                  dk.data_ptr(), dv.data_ptr(), _ptr(d_slopes), _ptr(w), size, on.ptr))
    return dq, dk, dv, d_slopes


def rotation_table(positions: int, rot: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """float32[positions, rot]: cosines, then sines, of position * base^(-2 i / rot), computed in 64 bits."""
    _want(positions > 0 and rot > 0 and rot % 16 == 0, "rot: a multiple of 16")
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


def _norm(q, k, q_weight, k_weight, pos, table, eps: float):
    dev, dtype = q.device, q.dtype
    _want(dtype in _DTYPE, "q and k: float32, float16 or bfloat16")
    strides = _heads_of(q, "q", dtype, dev) + _heads_of(k, "k", dtype, dev)
    tokens, heads, dim = q.shape
    _want(k.shape[0] == tokens and k.shape[2] == dim, "k: [tokens, kv_heads, dim], as many tokens and elements as q")
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        _want(w.dtype == torch.float32 and w.device == dev and w.is_contiguous() and w.numel() == dim and w.data_ptr() % 16 == 0,
              f"{name}: float32[dim], aligned to 16 bytes")
    _ints(pos, tokens, dev, "pos")
    rot = n_pos = 0
    if table is not None:
        _want(table.dtype == torch.float32 and table.device == dev and table.is_contiguous() and table.dim() == 2 and table.data_ptr() % 16 == 0 and
              pos is not None, "table: float32[positions, rot], aligned to 16 bytes, and pos with it")
        n_pos, rot = table.shape
    return dev, _Heads(q.data_ptr(), k.data_ptr(), *strides, tokens, heads, k.shape[1], dim, _DTYPE[dtype], q_weight.data_ptr(),
                       k_weight.data_ptr(), _ptr(pos), rot, n_pos, _ptr(table), eps)


def norm_rotate(q, k, q_weight, k_weight, pos=None, table=None, eps: float = 1e-6, stream=None):
    """RMS norm of every head of q [tokens, heads, dim] and k [tokens, kv_heads, dim] with weights (float32[dim]), and the rotation of its first
    table.shape[1] elements by the token's position (rotation_table); new tensors (q, k), rows end to end.  dim: a multiple of 8 up to 256.
    Rows of a negative pos have no token and become zeros; those of a position beyond the table become NaN."""
    L = load_library()
    dev, h = _norm(q, k, q_weight, k_weight, pos, table, eps)
    with _On(dev, stream) as on:
        q_out, k_out = torch.empty(q.shape, dtype=q.dtype, device=dev), torch.empty(k.shape, dtype=k.dtype, device=dev)
        _ok(L.lgp_norm_rotate(on.index, C.byref(h), q_out.data_ptr(), k_out.data_ptr(), on.ptr))
    return q_out, k_out


def norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, pos=None, table=None, eps: float = 1e-6, stream=None):
    """Gradients (dq, dk, dq_weight, dk_weight) of norm_rotate, from those of its results; the other arguments are what it was given."""
    L = load_library()
    dev, h = _norm(q, k, q_weight, k_weight, pos, table, eps)
    with _On(dev, stream) as on:
        dq_out, dk_out = _like(dq_out, q.shape, "dq_out", q.dtype, dev), _like(dk_out, k.shape, "dk_out", k.dtype, dev)
        dq, dk = torch.empty(q.shape, dtype=q.dtype, device=dev), torch.empty(k.shape, dtype=k.dtype, device=dev)
        dqw, dkw = torch.empty_like(q_weight), torch.empty_like(k_weight)
        w, size = _workspace(on, dev, L.lgp_norm_rotate_workspace, C.byref(h))
        _ok(L.lgp_norm_rotate_backward(on.index, C.byref(h), dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(), dk.data_ptr(), dqw.data_ptr(),
                                       dkw.data_ptr(), _ptr(w), size, on.ptr))
    return dq, dk, dqw, dkw


class PackedActivations:
    """Activations in 8 bits: values (int8[tokens, width rounded up to 16]) times 2^(exps - 127) (uint8[tokens, groups of 32])."""

    def __init__(self, values, exps, width: int, dtype, pos=None):
        _want(values.dim() == 2 and values.dtype == torch.int8 and values.is_contiguous() and values.is_cuda and values.data_ptr() % 16 == 0 and width > 0 and
              values.shape[1] == (width + 15) // 16 * 16, "values: contiguous int8[tokens, width rounded up to 16], on a GPU")
        _want(exps.dtype == torch.uint8 and exps.is_contiguous() and exps.device == values.device and
              tuple(exps.shape) == (values.shape[0], (width + 31) // 32), "exps: contiguous uint8[tokens, (width + 31) / 32]")
        _want(dtype in _DTYPE, "dtype: float32, float16 or bfloat16")
        _ints(pos, values.shape[0], values.device, "pos")
        self.values, self.exps, self.width, self.dtype, self.pos = values, exps, int(width), dtype, pos
        self.c = _Packed(values.shape[0], width, _DTYPE[dtype], values.data_ptr(), exps.data_ptr(), _ptr(pos))

    @property
    def shape(self):
        return (self.values.shape[0], self.width)


def _rows2(t, name: str):
    _want(t.dim() == 2 and t.is_cuda and (t.stride(1) == 1 or t.shape[1] == 1 or t.numel() == 0), f"{name}: [tokens, width] on a GPU, values of a row side by side")
    return t.stride(0)


def pack_activations(x, pos=None, stream=None) -> PackedActivations:
    """x [tokens, width] (float32, float16 or bfloat16, values of a row side by side) in 8 bits: 32 values of a row share a power of two.  Rows of a
    negative pos (int32[tokens]) hold no token: they are not read and packed as zeros."""
    L = load_library()
    row = _rows2(x, "x")
    _want(x.dtype in _DTYPE and x.shape[1] > 0, "x: float32, float16 or bfloat16, one value in a row at least")
    tokens, width = x.shape
    _ints(pos, tokens, x.device, "pos")
    with _On(x.device, stream) as on:
        values = torch.empty((tokens, (width + 15) // 16 * 16), dtype=torch.int8, device=x.device)
        exps = torch.empty((tokens, (width + 31) // 32), dtype=torch.uint8, device=x.device)
        packed = PackedActivations(values, exps, width, x.dtype, pos)
        _ok(L.lgp_pack_activations(on.index, x.data_ptr(), row, C.byref(packed.c), on.ptr))
    return packed


def unpack_activations(packed: PackedActivations, stream=None) -> torch.Tensor:
    """The values that `packed` stands for, in the type that came."""
    L = load_library()
    with _On(packed.values.device, stream) as on:
        x = torch.empty(packed.shape, dtype=packed.dtype, device=packed.values.device)
        _ok(L.lgp_unpack_activations(on.index, C.byref(packed.c), x.data_ptr(), on.ptr))
    return x


def packed_weight_grad(packed: PackedActivations, dy, bias: bool = True, stream=None):
    """(dw, db) of a linear layer y = x W^T + b whose input was packed: float32[out, width] and float32[out] (None if bias is False), from dy [tokens,
    out] in bfloat16, or in float16 if x was."""
    L = load_library()
    row = _rows2(dy, "dy")
    _want(dy.shape[0] == packed.shape[0] and dy.shape[1] > 0 and dy.device == packed.values.device, "dy: [tokens, out], where the packed rows are")
    _want(dy.dtype == torch.bfloat16 or (dy.dtype == torch.float16 and packed.dtype == torch.float16),
          "dy: bfloat16, or float16 with activations that came in float16")
    out = dy.shape[1]
    with _On(dy.device, stream) as on:
        dw = torch.empty((out, packed.width), dtype=torch.float32, device=dy.device)
        db = torch.empty(out, dtype=torch.float32, device=dy.device) if bias else None
        w, size = _workspace(on, dy.device, L.lgp_packed_weight_grad_workspace, C.byref(packed.c), out)
        _ok(L.lgp_packed_weight_grad(on.index, C.byref(packed.c), dy.data_ptr(), row, _DTYPE[dy.dtype], out, dw.data_ptr(), _ptr(db), _ptr(w), size, on.ptr))
    return dw, db
