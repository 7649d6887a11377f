"""The operators of a model layer in 64 bits, one document, row or group at a time, with a bound on what the kernels' roundings may do to each result."""
from __future__ import annotations

import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a place of a rounded number
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}                   # what fp16 loses of the smallest numbers


def attention(q, k, v, docs, d_out=None, slopes=None, cap=0.0, scale=None, exact_delta=True):
    """docs: (q_off, q_len, k_off, k_len) per document; q_pos and k_pos in `docs` too if there are slopes.  Returns {name: (value, bound)} in
    float64.  Bounds add up: the rounding of the result, of the probabilities (dU) in the product that makes it, and the fp32 arithmetic before."""
    u, tiny = UNIT[q.dtype], TINY[q.dtype]
    H, D, K = q.shape[1], q.shape[2], k.shape[1]
    G, scale = H // K, D ** -0.5 if scale is None else scale
    f8 = dict(dtype=torch.float64, device=q.device)
    val = dict(out=torch.zeros(q.shape, **f8), lse=torch.full(q.shape[:2], -math.inf, **f8), dq=torch.zeros(q.shape, **f8),
               dk=torch.zeros(k.shape, **f8), dv=torch.zeros(k.shape, **f8), d_slopes=torch.zeros(H, **f8))
    tol = {n: torch.zeros_like(x) for n, x in val.items()}
    for qo, qn, ko, kn in docs["spans"]:
        if not qn or not kn:
            continue
        far = (docs["q_pos"][qo:qo + qn, None] - docs["k_pos"][None, ko:ko + kn]).abs().double() if slopes is not None else None
        for h in range(H):
            Q, X, Y = q[qo:qo + qn, h].double(), k[ko:ko + kn, h // G].double(), v[ko:ko + kn, h // G].double()
            z0 = scale * Q @ X.T
            z = cap * torch.tanh(z0 / cap) if cap else z0
            size = abs(scale) * Q.abs() @ X.abs().T * (D / 4 + 8) + (cap * 8 if cap else 0)        # of a score's error, in 2^-24: products, cap
            if slopes is not None:
                z = z - slopes[h].double() * far
                size = size + 4 * slopes[h].abs().double() * far
            ez = 2.0 ** -24 * (size + 4 * z.abs() + 16).max()            # relative error of a probability
            lse = torch.logsumexp(z, 1)
            P = torch.exp(z - lse[:, None])
            O = P @ Y
            val["out"][qo:qo + qn, h], val["lse"][qo:qo + qn, h] = O, lse
            tol["out"][qo:qo + qn, h] = u * O.abs() + (u + 3 * ez) * P @ Y.abs() + tiny * (Y.abs().sum(0) + 1)
            tol["lse"][qo:qo + qn, h] = 2 * ez + 2.0 ** -22 * lse.abs()
            if d_out is None:
                continue
            g = d_out[qo:qo + qn, h].double()
            dP, delta = g @ Y.T, (g * O).sum(1, keepdim=True)
            dS = P * (dP - delta)
            dU = dS * (1 - (z0 / cap).tanh() ** 2) if cap else dS
            # error of dS: probabilities, and delta from a rounded out (without what the rounding took off) with probabilities rounded to u
            size = g.abs() @ Y.abs().T + g.abs() @ (P @ Y.abs()).T.abs().max(1).values[:, None]
            e_delta = (u + (2.0 ** -2 * u if exact_delta else u)) * (g.abs() * (P @ Y.abs())).sum(1, keepdim=True)
            eS = P * ((4 * ez + 2.0 ** -18) * size + e_delta)
            val["dq"][qo:qo + qn, h] = scale * dU @ X
            tol["dq"][qo:qo + qn, h] = u * (scale * dU @ X).abs() + abs(scale) * (u * dU.abs() + eS + tiny) @ X.abs() + tiny
            val["dk"][ko:ko + kn, h // G] += scale * dU.T @ Q
            tol["dk"][ko:ko + kn, h // G] += abs(scale) * (u * dU.abs() + eS + tiny).T @ Q.abs() + tiny
            val["dv"][ko:ko + kn, h // G] += P.T @ g
            tol["dv"][ko:ko + kn, h // G] += (u + 4 * ez) * P.T @ g.abs() + tiny * 2.0 ** -11 * g.abs().sum(0) + tiny
            if slopes is not None:
                val["d_slopes"][h] -= (dS * far).sum()
                tol["d_slopes"][h] += ((16 * ez + 2.0 ** -18) * P * size * (far + (P * far).sum(1, keepdim=True))).sum()
    for n in ("dk", "dv"):
        tol[n] += u * val[n].abs()
    return {n: (val[n], tol[n]) for n in val}


def check(got, ref, what=""):
    val, tol = ref
    got = got.double()
    assert got.shape == val.shape, f"{what}: {tuple(got.shape)} instead of {tuple(val.shape)}"
    assert torch.equal(torch.isnan(got), torch.isnan(val)), f"{what}: NaN elsewhere"
    inf = torch.isinf(val)
    assert torch.equal(got[inf], val[inf]) and not torch.isinf(got[~inf]).any(), f"{what}: infinities elsewhere"
    ok = ~inf & ~torch.isnan(val)
    off = (got - val).abs()[ok] - tol[ok]
    assert off.numel() == 0 or off.max() <= 0, (f"{what}: {int((off > 0).sum())} of {off.numel()} beyond the bound, worst by "
                                                f"{float(off.max()):.3g} where {float(tol[ok][off.argmax()]):.3g} is allowed")


def head_norm(x, w, pos, table, eps, d_out=None):
    """RMS norm, weights and rotation of x [tokens, heads, dim]; {name: (value, bound)}."""
    u, tiny = UNIT[x.dtype], TINY.get(x.dtype, 0.0)
    D = x.shape[2]
    rot = 0 if table is None else table.shape[1]
    live = torch.ones(x.shape[0], dtype=torch.bool, device=x.device) if pos is None else pos >= 0
    X = torch.where(live[:, None, None], x.double(), 0.0)
    r = 1 / torch.sqrt((X * X).mean(2, keepdim=True) + eps)
    n = X * r
    W = w.double()

    def turn(y, back):
        if not rot:
            return y, y.abs()
        known = pos < table.shape[0]
        t = table[torch.where(live & known, pos, 0).long()].double()[:, None]
        c, s = t[..., :rot // 2], t[..., rot // 2:] * (-1 if back else 1)
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        y2 = torch.cat([a * c - b * s, b * c + a * s, y[..., rot:]], 2)
        size = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs(), y[..., rot:].abs()], 2)
        y2 = torch.where((live & ~known)[:, None, None], math.nan, y2)
        return torch.where(live[:, None, None], y2, 0.0), size

    e = 2.0 ** -24 * (D / 8 + 24)                 # of a norm: the sum of squares, the root and three products
    y, size = turn(n * W, False)
    ref = {"out": (y, u * y.abs() + e * size + tiny)}
    if d_out is not None:
        g0, size0 = turn(torch.where(live[:, None, None], d_out.double(), 0.0), True)
        g, sg = g0 * W, size0 * W.abs()
        m, sm = (g * n).mean(2, keepdim=True), (sg * n.abs()).mean(2, keepdim=True)
        dx = r * (g - n * m)
        ref["dx"] = (dx, u * dx.abs() + 3 * e * r * (sg + n.abs() * sm) + tiny)
        rows = x.shape[0] * x.shape[1]
        ref["dw"] = ((g0 * n).sum((0, 1)), (2.0 ** -24 * min(rows, 4096) + 2 * e) * (size0 * n.abs()).sum((0, 1)))
    return ref


def pack(x, pos=None):
    """The rule of the packed form, group by group: (values int8, exps uint8, the numbers they stand for in float64)."""
    T, W = x.shape
    values, exps, held = torch.zeros(T, (W + 15) // 16 * 16, dtype=torch.int8), torch.zeros(T, (W + 31) // 32, dtype=torch.uint8), torch.zeros(T, W, dtype=torch.float64)
    least = -24 if x.dtype == torch.float16 else -126
    X = x.double().cpu()
    for t in range(T):
        for g in range(0, W, 32):
            part = X[t, g:g + 32] if pos is None or int(pos[t]) >= 0 else torch.zeros(min(32, W - g), dtype=torch.float64)
            if not torch.isfinite(part).all():
                exps[t, g // 32], held[t, g:g + 32] = 255, math.nan
                continue
            top = float(part.abs().max())
            e = max(math.frexp(top)[1] - 1 - 6 if top else least, least)
            n = torch.tensor([round(float(a) / 2.0 ** e) for a in part], dtype=torch.float64).clamp(-127, 127)        # round(): ties to even
            values[t, g:g + n.numel()], exps[t, g // 32], held[t, g:g + 32] = n.to(torch.int8), e + 127, n * 2.0 ** e
    return values, exps, held
