"""What a layer has around its attention, in 64 bits, with a bound on what the kernels' roundings may do to each result."""
from __future__ import annotations

import math

import torch

from layer_common import TINY, UNIT

E = 2.0 ** -24


def live_rows(tokens, pos, device):
    return torch.ones(tokens, dtype=torch.bool, device=device) if pos is None else pos >= 0


def add_norm(x, residual, weight, pos, eps, dy=None, d_total=None, total=None):
    """{name: (value, bound)}.  The total is rounded from a sum in 32 bits (given, where it is not the subject); all else is of the rounded total.  A row's
    sums are taken by lanes of at most 32 elements each and joined in a tree of ten levels at most: 64 roundings, half of which a root leaves; a
    product or quotient adds one."""
    live = live_rows((x if x is not None else total).shape[0], pos, weight.device)[:, None]
    if total is None:
        total = x if residual is None else torch.where(live, x.to(torch.promote_types(x.dtype, torch.float32)) + residual, 0.0).to(residual.dtype)
    t, w = torch.where(live, total.double(), 0.0), weight.double()
    r = 1 / torch.sqrt((t * t).mean(1, keepdim=True) + eps)
    r = torch.where(live, r, 0.0)
    n = t * r
    ref = {"total": total, "r": r}
    if x is not None:
        u, tiny = UNIT[x.dtype], TINY[x.dtype]
        ref["y"] = (n * w, (u + 40 * E) * (n * w).abs() + tiny)
        ref["y32"] = (n * w, 40 * E * (n * w).abs())
    if dy is not None:
        g0 = torch.where(live, dy.double(), 0.0)
        dt = torch.where(live, d_total.double(), 0.0) if d_total is not None else torch.zeros_like(t)
        g = g0 * w
        mean, size = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
        d = dt + r * (g - n * mean)
        off = E * (dt.abs() + 48 * r * g.abs() + 112 * r * n.abs() * size)
        for name, dtype in (("dx", dy.dtype), ("d_residual", total.dtype)):
            ref[name] = (d, UNIT[dtype] * d.abs() + off + TINY[dtype])
        # a lane adds its rows one by one, of which a workgroup has T / 1024 or fewer than as many more, and 1024 workgroups at most are added by 32
        rows = t.shape[0]
        ref["dw"] = ((g0 * n).sum(0), E * (min(rows, rows / 1024 + 1) + 32 + 32 + 45) * (g0 * n).abs().sum(0))
    return ref


def rows8(y, tol, values, scales, live):
    """Checks rows in 8 bits against the 64-bit numbers that they stand for, known to `tol`."""
    width = y.shape[1]
    assert values.shape[1] == (width + 15) // 16 * 16 and (values[:, width:] == 0).all()
    v, s = values[:, :width].double(), scales.double()
    assert (v[~live] == 0).all() and (s[~live] == 0).all()
    odd = live & ~torch.isfinite(y).all(1)
    assert torch.isnan(s[odd]).all() and (v[odd] == 0).all()
    y, tol, v, s = y[live & ~odd], tol[live & ~odd], v[live & ~odd], s[live & ~odd]
    if not y.numel():
        return
    top, least = y.abs().amax(1), 2.0 ** -126
    want = (top / 127).clamp(min=least)
    assert ((s - want).abs() <= tol.amax(1) / 127 + 2 * E * want).all()
    assert (v.abs().amax(1)[top / 127 >= 2 * least] == 127).all()
    # half a step, and what the rounding of the step's reciprocal and of the product may add to a number of up to 127
    assert ((v * s[:, None] - y).abs() <= s[:, None] * (0.5 + 127 * 3 * E) + tol).all()


def clip(grads, most):
    """(norm, the scaled gradients in 64 bits)."""
    norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))
    by = min(1.0, most / norm) if math.isfinite(norm) and norm > 0 else 1.0
    return norm, [g.double() * by for g in grads]
