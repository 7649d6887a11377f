"""Performance cases of the operators that a model layer over sampled neighbourhoods is made of.

A document is a run of rows of a token matrix: a frontier vertex and its samples as the sampler's fixed-width lists have them
(a slot without a sample holds no token, and its row holds anything, NaN too), a whole sampled neighbourhood packed end to end, or
a long list that single vertices are compared with.  `op` names the calls one pass makes:

  attend        attention inside documents: softmax of cap * tanh(scale * q.k / cap) - slope * |position difference|
  attend_train  the same and its gradients by q, k, v and the slopes
  rotate        RMS norm of every query and key head with weights, and the rotation by the token's position
  rotate_train  the same and its gradients by q, k and the weights
  pack          activations to 8 bits (a power of two per 32 values of a row) and back
  pack_train    activations to 8 bits, and the gradients of a linear layer's weights and bias from them

Types are named fp32, fp16 and bf16.  Values are standard normal draws unless a comment says otherwise.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
POSITIONS = 8192          # rows of the rotation table
GROUP = 32                # values that share a power of two

# docs, q_len and k_len (rows that each document owns; shared: queries and keys are the same rows), ragged (documents have 0 to that
# many tokens), slots (documents lie k_len rows apart whatever they hold, else packed end to end), heads / kv_heads / dim, cap (0: none),
# bias (slopes by head), hops (positions are hop numbers 0, 1, 2, else places)
_ATTEND = dict(op="attend", docs=1, q_len=1, k_len=1, shared=False, ragged=False, slots=False, heads=4, kv_heads=4, dim=64, dtype="bf16", cap=0.0,
               bias=False, hops=True)
# tokens, heads / kv_heads / dim, rot (dimensions that are rotated), absent (share of rows without a token)
_ROTATE = dict(op="rotate", tokens=1, heads=4, kv_heads=4, dim=64, rot=64, dtype="bf16", absent=0.0)
# tokens, width of the activations, out (rows of the weight), absent as above
_PACK = dict(op="pack", tokens=1, width=128, out=0, dtype="fp16", absent=0.0)


def listed():
    return [
        # One vertex of a request against its neighbourhood of fan-outs 25 and 10: latency.
        dict(_ATTEND, name="attend_one", k_len=276, cap=30.0, bias=True),
        # Sixteen single queries against long lists, two key heads for sixteen query heads: reads the lists once.
        dict(_ATTEND, name="attend_lists", docs=16, k_len=50_001, heads=16, kv_heads=2, dim=128),
        # Second hop of a batch of 8192 seeds, fan-outs 15 and 10: every frontier vertex over its own samples, hidden size 256.
        dict(_ATTEND, name="attend_samples_train", op="attend_train", docs=122_880, k_len=10, ragged=True, slots=True, heads=8, kv_heads=8, dim=32,
             dtype="fp16"),
        # A batch of 1024 seeds, each with its whole neighbourhood of fan-outs 25 and 10 in slots, scores capped and falling with the hops.
        dict(_ATTEND, name="attend_hoods_train", op="attend_train", docs=1024, q_len=276, k_len=276, shared=True, ragged=True, slots=True, heads=8,
             kv_heads=8, dim=32, cap=30.0, bias=True),
        # Neighbourhoods of 1 + 15 + 150 + 750 vertices, packed, half as many key heads: an ordinary forward pass.
        dict(_ATTEND, name="attend_packed", docs=256, q_len=916, k_len=916, shared=True, ragged=True, heads=4, kv_heads=2, dim=64, dtype="fp16", cap=50.0),
        # Four long lists attended in full with a bias by place: the largest.
        dict(_ATTEND, name="attend_long_train", op="attend_train", docs=4, q_len=8192, k_len=8192, shared=True, heads=8, kv_heads=4, dim=128, bias=True,
             hops=False),
        # The queries and keys of one request's neighbourhood: latency.
        dict(_ROTATE, name="rotate_one", tokens=276),
        # Those of a batch of neighbourhoods in slots, forward and backward, hidden size 256.
        dict(_ROTATE, name="rotate_hoods_train", op="rotate_train", tokens=282_624, heads=8, kv_heads=8, dim=32, rot=16, absent=0.3),
        # Wide heads of a long packed list, grouped keys.
        dict(_ROTATE, name="rotate_wide", tokens=500_000, heads=8, kv_heads=2, dim=128, rot=128, dtype="fp16"),
        # The features of a smallest batch, rows that are no multiple of a group.
        dict(_PACK, name="pack_small", tokens=1024, width=100, dtype="fp32"),
        # Features of 1024 values, as wide ones are extracted for 4096 seeds, with a layer of 256 on them.
        dict(_PACK, name="pack_wide_train", op="pack_train", tokens=400_000, width=1024, out=256),
        # Hidden activations of 256 values of a large batch, slots without tokens among them.
        dict(_PACK, name="pack_hidden_train", op="pack_train", tokens=1_000_003, width=256, out=256, dtype="bf16", absent=0.3),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {c["op"].split("_")[0]: work(c) for c in sorted(listed(), key=lambda c: work(c)["flops"])}
    while True:
        op = rng.choice(["attend", "attend_train", "rotate", "rotate_train", "pack", "pack_train"])
        if op.startswith("attend"):
            kv = rng.choice([1, 2, 4, 8])
            c = dict(_ATTEND, op=op, heads=kv * rng.choice([1, 1, 2, 4]), kv_heads=kv, dim=8 * rng.randint(2, 16), dtype=rng.choice(["fp16", "bf16"]),
                     cap=rng.choice([0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.5, hops=rng.random() < 0.5)
            form = rng.choice(["single", "samples", "packed", "packed"])
            if form == "single":           # one query per document; a third of them over long lists
                c.update(docs=log(1, 64), k_len=log(1, 60_000), slots=rng.random() < 0.5)
            elif form == "samples":        # a frontier over its samples
                c.update(docs=log(1000, 120_000), k_len=rng.randint(2, 32), ragged=True, slots=True)
            else:                          # documents that attend to themselves
                length = log(2, 8192)
                c.update(docs=log(1, max(1, min(2000, 400_000 // length))), q_len=length, k_len=length, shared=True, ragged=rng.random() < 0.6,
                         slots=rng.random() < 0.5)
            if c["docs"] * c["heads"] * c["q_len"] * c["k_len"] > 1 << 31 or c["docs"] * c["k_len"] * c["heads"] * c["dim"] > 1 << 30:
                continue
        elif op.startswith("rotate"):
            kv = rng.choice([1, 2, 4, 8])
            dim = 8 * rng.randint(2, 32)
            c = dict(_ROTATE, op=op, tokens=log(1, 600_000), heads=kv * rng.choice([1, 2, 4]), kv_heads=kv, dim=dim, rot=16 * rng.randint(0, dim // 16),
                     dtype=rng.choice(["fp32", "fp16", "bf16"]), absent=rng.choice([0.0, 0.3]))
        else:
            c = dict(_PACK, op=op, tokens=log(1, 1_000_000), width=log(8, 1024), dtype=rng.choice(["fp32", "fp16", "bf16"]), absent=rng.choice([0.0, 0.3]))
            if op == "pack_train":
                c.update(out=log(8, 1024), dtype=rng.choice(["fp16", "bf16"]))
        w, top = work(c), most[op.split("_")[0]]
        if w["bytes"] <= top["bytes"] * 1.5 and w["flops"] <= top["flops"]:
            return c


def _documents(c, g):
    """Offsets, token counts (None: all rows) and positions of a case's queries or keys, by the side's length."""
    def side(length):
        n = c["docs"]
        if not c["ragged"]:
            return torch.arange(n + 1, dtype=torch.int32, device="cuda") * length, None, n * length
        lens = (torch.randperm(n, generator=g, device="cuda") * (length + 1) // n).to(torch.int32)      # every length alike, in any order
        if c["slots"]:
            return torch.arange(n + 1, dtype=torch.int32, device="cuda") * length, lens, n * length
        offs = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        offs[1:] = lens.cumsum(0)
        return offs, None, int(offs[-1])

    def places(offs, total, keys):
        # the place of a row inside its document; as hop numbers the first row, the next 25 and the others; a single query is the vertex itself
        row = torch.arange(total, dtype=torch.int32, device="cuda")
        at = row - offs[torch.searchsorted(offs[1:], row, right=True)]
        if c["hops"]:
            at = (at > 0).int() + (at > 25).int()
            return at + 1 if keys and not c["shared"] else at
        return at

    k_offs, k_lens, k_total = side(c["k_len"])
    if c["shared"]:
        q_offs, q_lens, q_total = k_offs, k_lens, k_total
    else:
        q_offs, q_lens, q_total = torch.arange(c["docs"] + 1, dtype=torch.int32, device="cuda") * c["q_len"], None, c["docs"] * c["q_len"]
    return q_offs, q_lens, q_total, places(q_offs, q_total, False), k_offs, k_lens, k_total, places(k_offs, k_total, True)


def prepare(case, seed):
    c, g = dict(case), torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TYPES[c["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    if c["op"].startswith("attend"):
        q_offs, q_lens, q_total, q_pos, k_offs, k_lens, k_total, k_pos = _documents(c, g)
        H, K, D = c["heads"], c["kv_heads"], c["dim"]
        s = dict(q=normal(q_total, H, D), k=normal(k_total, K, D), v=normal(k_total, K, D), d_out=normal(q_total, H, D), q_offs=q_offs, k_offs=k_offs,
                 q_lens=q_lens, k_lens=k_lens, q_pos=q_pos, k_pos=k_pos, slopes=None)
        if c["bias"]:                       # geometric over the heads, and not quite the same in every run of a training
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H) * (1 + 0.1 * torch.rand(H, generator=g, device="cuda"))
        for lens, offs, names in ((q_lens, q_offs, ("q", "d_out")), (k_lens, k_offs, ("k", "v"))):
            if lens is not None:            # a slot without a sample holds what was there before
                row = torch.arange(s[names[0]].shape[0], dtype=torch.int32, device="cuda")
                doc = torch.searchsorted(offs[1:], row, right=True)
                for name in names:
                    s[name][row - offs[doc] >= lens[doc]] = float("nan")
    elif c["op"].startswith("rotate"):
        T, H, K, D, R = c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rot"]
        qkv = normal(T, H + 2 * K, D)       # as one product leaves queries, keys and values
        pos = torch.randint(0, POSITIONS, (T,), generator=g, device="cuda", dtype=torch.int32)
        pos[torch.rand(T, generator=g, device="cuda") < c["absent"]] = -1
        qkv[pos < 0] = float("nan")
        angle = torch.arange(POSITIONS, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / max(R, 1))
        s = dict(qkv=qkv, pos=pos, table=torch.cat([angle.cos(), angle.sin()], 1).float() if R else None,
                 q_weight=1 + 0.2 * normal(D, dtype=torch.float32), k_weight=1 + 0.2 * normal(D, dtype=torch.float32), dq=normal(T, H, D), dk=normal(T, K, D))
    else:
        T, W = c["tokens"], c["width"]
        # rows and channels of different sizes, as activations have them
        x = torch.randn((T, W), generator=g, device="cuda") * torch.exp(0.5 * torch.randn((1, W), generator=g, device="cuda"))
        pos = torch.zeros(T, dtype=torch.int32, device="cuda")
        if c["absent"]:
            pos[torch.rand(T, generator=g, device="cuda") < c["absent"]] = -1
        x[pos < 0] = float("nan")
        s = dict(x=x.to(dt), pos=pos if c["absent"] else None, dy=None)
        if c["op"] == "pack_train":
            s["dy"] = normal(T, c["out"])
            if c["absent"]:
                s["dy"][pos < 0] = float("nan")
    s["case"] = c
    return s


def run(s):
    c = s["case"]
    if own:
        return _run_own(s)
    if c["op"].startswith("attend"):
        return _attend_plain(s)
    if c["op"].startswith("rotate"):
        return _rotate_plain(s)
    return _pack_plain(s)


def _run_own(s):
    import paper_2305_16588_amd as lgp
    c = s["case"]
    if c["op"].startswith("attend"):
        train = c["op"] == "attend_train"
        docs = lgp.Documents(s["q_offs"], s["k_offs"], q_lens=s["q_lens"], k_lens=s["k_lens"], q_pos=s["q_pos"], k_pos=s["k_pos"])
        out, lse, rest = lgp.attend(s["q"], s["k"], s["v"], docs, slopes=s["slopes"], cap=c["cap"], rest=train)
        if not train:
            return [out, lse]
        return [out, lse, *lgp.attend_backward(s["d_out"], s["q"], s["k"], s["v"], out, lse, docs, rest=rest, slopes=s["slopes"], cap=c["cap"])]
    if c["op"].startswith("rotate"):
        q, k = s["qkv"][:, :c["heads"]], s["qkv"][:, c["heads"]:c["heads"] + c["kv_heads"]]
        rest = (s["q_weight"], s["k_weight"], s["pos"], s["table"])
        got = lgp.norm_rotate(q, k, *rest)
        return [*got, *lgp.norm_rotate_backward(s["dq"], s["dk"], q, k, *rest)] if c["op"] == "rotate_train" else list(got)
    packed = lgp.pack_activations(s["x"], pos=s["pos"])
    return list(lgp.packed_weight_grad(packed, s["dy"])) if c["op"] == "pack_train" else [lgp.unpack_activations(packed)]


def _rows(offs, lens, length, total):
    """Rows of each document, padded to `length`, and which of them hold a token."""
    at = torch.arange(length, device=offs.device)
    has = offs[1:] - offs[:-1] if lens is None else lens
    return (offs[:-1, None] + at).clamp(max=max(total - 1, 0)).long(), at < has[:, None]


def _attend_plain(s):
    c = s["case"]
    n, H, K, D, Lq, Lk = c["docs"], c["heads"], c["kv_heads"], c["dim"], c["q_len"], c["k_len"]
    G, cap, scale = H // K, c["cap"], c["dim"] ** -0.5
    dt, Tq, Tk = s["q"].dtype, s["q"].shape[0], s["k"].shape[0]
    q_row, q_has = _rows(s["q_offs"], s["q_lens"], Lq, Tq)
    k_row, k_has = _rows(s["k_offs"], s["k_lens"], Lk, Tk)

    def queries(x):     # [Tq, H, D] -> [n * K, Lq * G, D]
        if not Tq:
            return torch.zeros(n * K, Lq * G, D, device=x.device)
        return torch.where(q_has[:, :, None, None], x[q_row].float(), 0.0).view(n, Lq, K, G, D).permute(0, 2, 1, 3, 4).reshape(n * K, Lq * G, D)

    def keys(x):        # [Tk, K, D] -> [n * K, Lk, D]
        if not Tk:
            return torch.zeros(n * K, Lk, D, device=x.device)
        return torch.where(k_has[:, :, None, None], x[k_row].float(), 0.0).permute(0, 2, 1, 3).reshape(n * K, Lk, D)

    def back(x, width, row, has, total):      # the other way, zeros where no token is
        full = torch.zeros(total, width, *x.shape[3:], device=x.device)
        full[row[has]] = x.reshape(x.shape[0], x.shape[1], width, *x.shape[3:])[has]
        return full

    q, k, v = queries(s["q"]), keys(s["k"]), keys(s["v"])
    z = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale)
    t = torch.tanh(z / cap) if cap else None
    z = t * cap if cap else z
    far = None
    if s["slopes"] is not None:
        far = (s["q_pos"][q_row][:, :, None] - s["k_pos"][k_row][:, None, :]).abs().float()                # [n, Lq, Lk]
        z = (z.view(n, K, Lq, G, Lk) - s["slopes"].view(1, K, 1, G, 1) * far[:, None, :, None, :]).view(n * K, Lq * G, Lk)
    seen = k_has[:, None, :].expand(n, K, Lk).reshape(n * K, 1, Lk)
    z = z.masked_fill_(~seen, -math.inf)
    top = z.amax(2, keepdim=True) if Lk else torch.full((n * K, Lq * G, 1), -math.inf, device=z.device)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(z - top)
    del z
    total = p.sum(2, keepdim=True)
    lse = torch.log(total) + top
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.bmm(p, v)

    def out_rows(x):        # [n * K, Lq * G, D] -> [n, Lq, K * G, D]
        return x.view(n, K, Lq, G, -1).permute(0, 2, 1, 3, 4).reshape(n, Lq, H, -1)

    out = back(out_rows(o), H, q_row, q_has, Tq).to(dt)
    lse_full = torch.full((Tq, H), -math.inf, device=o.device)
    lse_full[q_row[q_has]] = out_rows(lse)[..., 0][q_has]
    if c["op"] == "attend":
        return [out, lse_full]
    do = queries(s["d_out"])
    dv = torch.bmm(p.transpose(1, 2).contiguous(), do)
    ds = torch.bmm(do, v.transpose(1, 2).contiguous())
    ds = ds.sub_((do * o).sum(2, keepdim=True)).mul_(p)
    del p
    d_slopes = None
    if far is not None:
        d_slopes = -(ds.view(n, K, Lq, G, Lk) * far[:, None, :, None, :]).sum((4, 2, 0)).view(H)
    if cap:
        ds = ds * (1 - t * t)
    dq = torch.bmm(ds, k).mul_(scale)
    dk = torch.bmm(ds.transpose(1, 2).contiguous(), q).mul_(scale)

    def key_rows(x):
        return x.view(n, K, Lk, D).permute(0, 2, 1, 3)

    return [out, lse_full, back(out_rows(dq), H, q_row, q_has, Tq).to(dt), back(key_rows(dk), K, k_row, k_has, Tk).to(dt),
            back(key_rows(dv), K, k_row, k_has, Tk).to(dt), d_slopes]


def _rotate_plain(s, eps=1e-6):
    c = s["case"]
    H, K, R = c["heads"], c["kv_heads"], c["rot"]
    has = (s["pos"] >= 0)[:, None, None]
    turn = s["table"][s["pos"].clamp(min=0).long()][:, None, :] if R else None

    def rotate(x, back):
        if not R:
            return x
        cos, sin = turn[..., :R // 2], turn[..., R // 2:]
        a, b = x[..., :R // 2], x[..., R // 2:R]
        sin = -sin if back else sin
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., R:]], -1)

    def forward(x, w):
        x = torch.where(has, x.float(), 0.0)
        return torch.where(has, rotate(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w, False), 0.0).to(s["qkv"].dtype)

    def backward(dy, x, w):
        x, dy = torch.where(has, x.float(), 0.0), torch.where(has, rotate(dy.float(), True), 0.0)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
        x = x * r
        g = dy * w
        return (r * (g - x * (g * x).mean(-1, keepdim=True))).to(s["qkv"].dtype), (dy * x).sum((0, 1))

    q, k = s["qkv"][:, :H], s["qkv"][:, H:H + K]
    got = [forward(q, s["q_weight"]), forward(k, s["k_weight"])]
    if c["op"] == "rotate":
        return got
    (dq, dwq), (dk, dwk) = backward(s["dq"], q, s["q_weight"]), backward(s["dk"], k, s["k_weight"])
    return [*got, dq, dk, dwq, dwk]


def _pack_plain(s):
    x = s["x"].float()
    T, W = x.shape
    if s["pos"] is not None:
        x = torch.where((s["pos"] >= 0)[:, None], x, 0.0)
    x = torch.nn.functional.pad(x, (0, -W % GROUP)).view(T, -1, GROUP)
    top = x.abs().amax(2, keepdim=True)
    good = torch.isfinite(x).all(2, keepdim=True)
    least = -24 if s["x"].dtype == torch.float16 else -126
    # the largest value of a group lies in [64, 128) steps; what rounds to 128 is held as 127
    step = torch.ldexp(torch.ones_like(top), (torch.frexp(torch.where(good, top, 1.0)).exponent - 7).clamp(min=least))
    x = torch.where(good, (x / step).round().clamp(-127, 127) * step, math.nan).view(T, -1)[:, :W]
    if s["case"]["op"] == "pack":
        return [x.to(s["x"].dtype)]
    dy = s["dy"].float()
    if s["pos"] is not None:
        dy = torch.where((s["pos"] >= 0)[:, None], dy, 0.0)
    return [dy.t().contiguous() @ x, dy.sum(0)]


def work(case):
    c = case
    size = SIZE[c["dtype"]]
    if c["op"].startswith("attend"):
        n, H, K, D = c["docs"], c["heads"], c["kv_heads"], c["dim"]
        part, square = (0.5, 1 / 3) if c["ragged"] else (1.0, 1.0)
        tq, tk = n * c["q_len"] * (part if c["shared"] else 1.0), n * c["k_len"] * part
        pairs = n * c["q_len"] * c["k_len"] * (square if c["shared"] else part)
        rows_q, rows_k = n * c["q_len"] * (1.0 if c["slots"] or not c["shared"] else part), n * c["k_len"] * (1.0 if c["slots"] else part)
        b = (tq * H * D + 2 * tk * K * D) * size + rows_q * H * (D * size + 4)
        if c["op"] == "attend_train":       # q, k, v, out and its gradient again, and three gradients written
            b += (2 * tq * H * D + tq * H * 2 + 2 * tk * K * D) * size + (rows_q * H + 2 * rows_k * K) * D * size
        return {"bytes": b, "flops": pairs * H * D * (4 if c["op"] == "attend" else 14)}
    if c["op"].startswith("rotate"):
        rows = c["tokens"] * (c["heads"] + c["kv_heads"]) * c["dim"]
        has = 1 - c["absent"]
        b = rows * (has + 1) * size + c["tokens"] * 4
        if c["op"] == "rotate_train":
            b += rows * (2 * has + 1) * size + c["tokens"] * 4
        return {"bytes": b, "flops": rows * has * (8 if c["op"] == "rotate" else 24)}
    T, W, N, has = c["tokens"], c["width"], c["out"], 1 - c["absent"]
    packed = T * W * (1 + 1 / GROUP)
    if c["op"] == "pack":
        return {"bytes": T * W * (has * size + size) + 2 * packed, "flops": T * W * 6}
    return {"bytes": T * W * has * size + 2 * packed + T * N * has * size + 4 * N * (W + 1), "flops": T * W * 4 + 2 * T * has * W * N}


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"].startswith("attend"):
        return _attend_exact(s, c)
    if c["op"].startswith("rotate"):
        return _rotate_exact(s, c)
    return _pack_exact(s, c)


def _attend_exact(s, c):
    """Long documents one by one and head by head; many short ones as the list of all their pairs."""
    H, K, D, cap, train = c["heads"], c["kv_heads"], c["dim"], c["cap"], c["op"] == "attend_train"
    G, scale, dev = H // K, c["dim"] ** -0.5, s["q"].device
    q_at, k_at = s["q_offs"].long(), s["k_offs"].long()
    q_n = q_at[1:] - q_at[:-1] if s["q_lens"] is None else s["q_lens"].long()
    k_n = k_at[1:] - k_at[:-1] if s["k_lens"] is None else s["k_lens"].long()
    f8 = dict(dtype=torch.float64, device=dev)
    out, lse = torch.zeros(s["q"].shape, **f8), torch.full(s["q"].shape[:2], -math.inf, **f8)
    dq, dk, dv, d_slopes = torch.zeros(s["q"].shape, **f8), torch.zeros(s["k"].shape, **f8), torch.zeros(s["k"].shape, **f8), torch.zeros(H, **f8)
    if c["docs"] * (K if c["q_len"] * c["k_len"] > 1 << 20 else 1) > 4096:
        for lo in range(0, c["docs"], 4096):
            n = q_n[lo:lo + 4096] * k_n[lo:lo + 4096]
            doc = torch.repeat_interleave(torch.arange(n.numel(), device=dev), n)
            nth = torch.arange(doc.numel(), device=dev) - (n.cumsum(0) - n)[doc]
            doc = doc + lo
            i, j = q_at[doc] + nth // k_n[doc], k_at[doc] + nth % k_n[doc]
            if not i.numel():
                continue
            if i.numel() * H * D > 1 << 31:
                return None
            head = torch.arange(H, device=dev) // G
            q, k, v = s["q"][i].double(), s["k"][j].double()[:, head], s["v"][j].double()[:, head]
            u = (q * k).sum(2) * scale
            t = torch.tanh(u / cap) if cap else None
            u = t * cap if cap else u
            far = (s["q_pos"][i] - s["k_pos"][j]).abs().double()[:, None]
            if s["slopes"] is not None:
                u = u - s["slopes"].double() * far
            first = int(i.min())
            span = int(i.max()) - first + 1
            at = (i - first)[:, None].expand(-1, H)
            top = torch.full((span, H), -math.inf, **f8).scatter_reduce(0, at, u, "amax")
            e = torch.exp(u - top[i - first])
            total = torch.zeros((span, H), **f8).index_add(0, i - first, e)
            p = e / total[i - first]
            lse[first:first + span] = torch.where(total > 0, torch.log(total) + top, -math.inf)
            out.index_add_(0, i, p[..., None] * v)
            if train:
                do = s["d_out"][i].double()
                dp = (do * v).sum(2)
                ds = p * (dp - torch.zeros((span, H), **f8).index_add(0, i - first, p * dp)[i - first])
                d_slopes -= (ds * far).sum(0)
                ds = ds * (1 - t * t) if cap else ds
                dq.index_add_(0, i, ds[..., None] * k * scale)
                dk.index_add_(0, j, (ds[..., None] * q * scale).view(-1, K, G, D).sum(2))
                dv.index_add_(0, j, (p[..., None] * do).view(-1, K, G, D).sum(2))
    else:
        for d, (a, m, b, n) in enumerate(zip(q_at.tolist(), q_n.tolist(), k_at.tolist(), k_n.tolist())):
            if not m or not n:
                continue
            far = (s["q_pos"][a:a + m, None] - s["k_pos"][None, b:b + n]).abs().double()
            at_once = max(1, (1 << 28) // (m * n))
            for h in range(0, H, at_once):
                heads = torch.arange(h, min(H, h + at_once), device=dev)
                q, k, v = (x.double().transpose(0, 1) for x in (s["q"][a:a + m, heads], s["k"][b:b + n, heads // G], s["v"][b:b + n, heads // G]))
                u = (q @ k.transpose(1, 2)) * scale
                t = torch.tanh(u / cap) if cap else None
                u = t * cap if cap else u
                if s["slopes"] is not None:
                    u = u - s["slopes"].double()[heads, None, None] * far
                lse[a:a + m, heads] = torch.logsumexp(u, 2).t()
                p = torch.softmax(u, 2)
                del u
                out[a:a + m, heads] = (p @ v).transpose(0, 1)
                if train:
                    do = s["d_out"][a:a + m, heads].double().transpose(0, 1)
                    dv[b:b + n].index_add_(1, heads // G, (p.transpose(1, 2) @ do).transpose(0, 1))
                    ds = do @ v.transpose(1, 2)
                    ds = p * (ds - (p * ds).sum(2, keepdim=True))
                    d_slopes[heads] -= (ds * far).sum((1, 2))
                    ds = ds * (1 - t * t) if cap else ds
                    dq[a:a + m, heads] = (ds @ k).transpose(0, 1) * scale
                    dk[b:b + n].index_add_(1, heads // G, (ds.transpose(1, 2) @ q).transpose(0, 1) * scale)
    return [out, lse, dq, dk, dv, d_slopes if s["slopes"] is not None else None] if train else [out, lse]


def _rotate_exact(s, c, eps=1e-6):
    H, K, R, T = c["heads"], c["kv_heads"], c["rot"], c["tokens"]
    rows = torch.nonzero(s["pos"] >= 0)[:, 0]
    half = R // 2
    turn = None
    if R:
        turn = torch.complex(s["table"][:, :half].double(), s["table"][:, half:].double())[s["pos"][rows].long()][:, None]

    def rotated(x, by):
        if not R:
            return x
        z = torch.complex(x[..., :half], x[..., half:R]) * by
        return torch.cat([z.real, z.imag, x[..., R:]], 2)

    def both(lo, hi, w, dy):
        x, w = s["qkv"][rows, lo:hi].double(), w.double()
        size = torch.sqrt((x ** 2).mean(2, keepdim=True) + eps)
        y = torch.zeros(T, hi - lo, c["dim"], dtype=torch.float64, device=x.device)
        y[rows] = rotated(x / size * w, turn)
        if c["op"] == "rotate":
            return y, None, None
        dy = rotated(dy[rows].double(), turn.conj() if R else None)
        dx = torch.zeros_like(y)
        dx[rows] = dy * w / size - x * (dy * w * x).mean(2, keepdim=True) / size ** 3
        return y, dx, (dy * x / size).flatten(0, 1).sum(0)

    q, dq, dwq = both(0, H, s["q_weight"], s["dq"])
    k, dk, dwk = both(H, H + K, s["k_weight"], s["dk"])
    return [q, k] if c["op"] == "rotate" else [q, k, dq, dk, dwq, dwk]


def _pack_exact(s, c):
    T, W = s["x"].shape
    least = -24 if c["dtype"] == "fp16" else -126
    dw = torch.zeros(c["out"], W, dtype=torch.float64, device="cuda") if c["out"] else None
    db = torch.zeros(c["out"], dtype=torch.float64, device="cuda") if c["out"] else None
    held = torch.zeros(T, W, dtype=torch.float64, device="cuda") if not c["out"] else None
    for lo in range(0, T, 1 << 17):
        hi = min(T, lo + (1 << 17))
        x = s["x"][lo:hi].double()
        here = torch.ones(hi - lo, dtype=torch.bool, device=x.device) if s["pos"] is None else s["pos"][lo:hi] >= 0
        x[~here] = 0.0
        for g in range(0, W, GROUP):
            part = x[:, g:g + GROUP]
            top = part.abs().max(1, keepdim=True).values
            e = torch.where(top > 0, torch.floor(torch.log2(torch.where(top > 0, top, 1.0))), -1000.0)
            e = e + (torch.exp2(e + 1) <= top).double() - (torch.exp2(e) > top).double()        # log2 may round across a power of two
            step = torch.exp2((e - 6).clamp(min=least))
            x[:, g:g + GROUP] = (part / step).round().clamp(-127, 127) * step
        if c["op"] == "pack":
            held[lo:hi] = x
        else:
            dy = torch.where(here[:, None], s["dy"][lo:hi].double(), 0.0)
            dw += dy.t() @ x
            db += dy.sum(0)
    return [held] if c["op"] == "pack" else [dw, db]
