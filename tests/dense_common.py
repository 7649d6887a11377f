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


def gated(x, w_gate, w_up, act, pos, dh=None):
    """{name: (value, bound)}.  Sums in 32 bits of K products: K / 8 + 16 roundings of the sum of their sizes at most.  An activation has an error of its argument's
    rounding (g^2 + |g| times E, relative) and a few of its own; its slope is below 1.13 and the slope's slope below 1."""
    u, tiny = UNIT[x.dtype], TINY[x.dtype]
    live = live_rows(x.shape[0], pos, x.device)[:, None]
    X, G, U = torch.where(live, x.double(), 0.0), w_gate.double(), w_up.double()
    g, v = X @ G.T, X @ U.T
    e = E * (X.shape[1] / 8 + 16)
    eg, ev = e * X.abs() @ G.abs().T, e * X.abs() @ U.abs().T
    if act == "silu":
        p = torch.sigmoid(g)
        slope = p + g * p * (1 - p)
    else:
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        slope = p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    a = g * p
    more = 2 * E * (g * g + g.abs() + 16)
    ea, es = 1.13 * eg + more * a.abs(), eg + more * (p + (slope - p).abs())
    h = a * v
    ref = {"h": (h, u * h.abs() + 1.01 * (ea * v.abs() + a.abs() * ev) + 4 * E * h.abs() + tiny)}
    if dh is None:
        return ref
    D = torch.where(live, dh.double(), 0.0)
    dg, du = D * v * slope, D * a
    e_dg = D.abs() * 1.01 * (ev * slope.abs() + v.abs() * es) + (u + 4 * E) * dg.abs() + tiny
    e_du = D.abs() * ea + (u + 4 * E) * du.abs() + tiny
    e_dg, e_du = torch.where(live, e_dg, 0.0), torch.where(live, e_du, 0.0)
    dx = dg @ G + du @ U
    e = E * (2 * G.shape[0] / 8 + 32)
    ref["dx"] = (dx, u * dx.abs() + e_dg @ G.abs() + e_du @ U.abs() + e * 1.01 * (dg.abs() @ G.abs() + du.abs() @ U.abs()) + tiny)
    e = E * (X.shape[0] / 8 + 32)
    for name, d, ed in (("dw_gate", dg, e_dg), ("dw_up", du, e_du)):
        w = d.T @ X
        ref[name] = (w, u * w.abs() + ed.T @ X.abs() + e * 1.01 * d.abs().T @ X.abs() + tiny)
    return ref
