"""Performance cases of what a layer over sampled neighbourhoods has around its attention, in training and in serving.

A token is a row of a matrix: a sampled vertex in its slot (a slot without a sample holds no token, its position is negative and its row holds
anything, NaN too), or a vertex of a request.  `op` names the calls one pass makes:

  norm          the residual's addition and the RMS norm of the sum
  norm_train    the same and its gradients by the branch, the residual and the weights
  product       product of rows in 8-bit integers with weights in 8-bit integers, a scale for each row and each channel, and a bias
  serve         the residual's addition and the norm with its result in 8 bits, and such a product with it
  gated         activation(x Wg^T) * (x Wu^T)
  gated_train   the same and its gradients by x and both weights
  clip          the norm of all gradients of a model, and the gradients scaled down to a largest norm, into buffers of the optimizer's

Types are named fp32, fp16 and bf16.  Values are standard normal draws unless a comment says otherwise.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
EPS = 1e-6
CLASSES = 47              # outputs of a classifier

# tokens, width, dtype of the branch and of the norm's result, stream: that of the residual, absent (share of rows without a token)
_NORM = dict(op="norm", tokens=1, width=256, dtype="bf16", stream="bf16", absent=0.0)
# tokens, width, out (channels), dtype of the result; serve: stream and absent as above
_PRODUCT = dict(op="product", tokens=1, width=256, out=256, dtype="bf16", stream="bf16", absent=0.0)
# tokens, width (a multiple of 8), hidden, act (silu or gelu), absent
_GATED = dict(op="gated", tokens=1, width=256, hidden=704, dtype="bf16", act="silu", absent=0.0)
# layers, width, hidden: of the model; dtype of the matrices' gradients, those of vectors are fp32; apart: every gradient begins at a multiple of 16
# bytes, else they lie end to end in a bucket; most: the largest norm
_CLIP = dict(op="clip", layers=1, width=128, hidden=352, dtype="fp32", apart=True, most=1.0)


def listed():
    return [
        # One request's neighbourhood of fan-outs 25 and 10: latency.
        dict(_NORM, name="norm_one", tokens=276),
        # A batch of 1024 such neighbourhoods in slots, hidden size 256.
        dict(_NORM, name="norm_hoods_train", op="norm_train", tokens=282_624, absent=0.3),
        # Wide rows, whose residual is kept in 32 bits: the largest norm.
        dict(_NORM, name="norm_stream_train", op="norm_train", tokens=400_000, width=1024, dtype="fp16", stream="fp32"),
        # One vertex through a wide projection: reads the weights once.
        dict(_PRODUCT, name="serve_one", op="serve", width=1024, out=4096),
        # Queries, keys and values of a batch of neighbourhoods in slots.
        dict(_PRODUCT, name="serve_hoods", op="serve", tokens=282_624, out=768, absent=0.3),
        # A long list of features whose width is no multiple of 16.
        dict(_PRODUCT, name="product_list", tokens=50_001, width=1000, out=1024, dtype="fp16"),
        # The same kind of product with wide rows and many channels: the largest.
        dict(_PRODUCT, name="product_wide", tokens=65_536, width=4096, out=4096),
        # One vertex of a request.
        dict(_GATED, name="gated_one", width=1024, hidden=4096),
        # A training step of a batch of neighbourhoods in slots, a hidden size that is not even.
        dict(_GATED, name="gated_hoods_train", op="gated_train", tokens=282_624, hidden=683, absent=0.3),
        # A training step with wide rows: the largest.
        dict(_GATED, name="gated_wide_train", op="gated_train", tokens=32_768, width=2048, hidden=8192, dtype="fp16", act="gelu"),
        # The gradients of one small layer: latency.
        dict(_CLIP, name="clip_layer"),
        # Those of a deep model, over 200 tensors in one bucket.
        dict(_CLIP, name="clip_model", layers=24, width=1280, hidden=3456, dtype="bf16", apart=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        w, top = work(c), most.setdefault(c["op"].split("_")[0].replace("serve", "product"), dict(bytes=0, flops=0))
        top.update({n: max(top[n], w[n]) for n in top})
    while True:
        op = rng.choice(["norm", "norm_train", "product", "serve", "gated", "gated_train", "clip"])
        tokens, absent = log(1, 400_000), rng.choice([0.0, 0.0, 0.3])
        if op.startswith("norm"):
            dtype = rng.choice(["fp32", "fp16", "bf16"])
            c = dict(_NORM, op=op, tokens=tokens, width=log(8, 8192), dtype=dtype, stream=rng.choice([dtype, "fp32"]), absent=absent)
        elif op in ("product", "serve"):
            dtype = rng.choice(["fp16", "bf16"])
            c = dict(_PRODUCT, op=op, tokens=tokens, width=log(16, 8192), out=log(8, 8192), dtype=dtype)
            if op == "serve":
                c.update(stream=rng.choice([dtype, "fp32"]), absent=absent)
        elif op.startswith("gated"):
            c = dict(_GATED, op=op, tokens=tokens, width=8 * log(2, 512), hidden=log(8, 8192), dtype=rng.choice(["fp16", "bf16"]), act=rng.choice(["silu", "gelu"]),
                     absent=absent)
        else:
            c = dict(_CLIP, layers=log(1, 32), width=log(16, 1536), hidden=log(32, 4096), dtype=rng.choice(["fp32", "fp16", "bf16"]), apart=rng.random() < 0.5,
                     most=rng.choice([0.1, 1.0, 1e6]))
        w, top = work(c), most[op.split("_")[0].replace("serve", "product")]
        if w["bytes"] <= top["bytes"] and w["flops"] <= top["flops"]:
            return c


def _gradients(c):
    """Shapes and types of a model's gradients."""
    w, h = c["width"], c["hidden"]
    layer = [((3 * w, w), c["dtype"]), ((w, w), c["dtype"]), ((h, w), c["dtype"]), ((h, w), c["dtype"]), ((w, h), c["dtype"]),
             ((w,), "fp32"), ((w,), "fp32"), ((32,), "fp32"), ((32,), "fp32")]
    return layer * c["layers"] + [((CLASSES, w), c["dtype"]), ((CLASSES,), "fp32")]


def _rows8(x):
    """Rows in 8-bit integers, filled up with zeros to a multiple of 16, and their scales."""
    scale = x.abs().amax(1) / 127
    v = (x / scale[:, None]).round().clamp(-127, 127).to(torch.int8)
    return torch.nn.functional.pad(v, (0, -x.shape[1] % 16)).contiguous(), scale


def prepare(case, seed):
    c, g = dict(case), torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    s = dict(case=c, pos=None)
    if c["op"] == "clip":
        shapes = _gradients(c)
        flat, at, places = {}, {}, []
        for shape, t in shapes:
            n = math.prod(shape)
            places.append((t, at.get(t, 0), shape, n))
            at[t] = at.get(t, 0) + (-(-n // 8) * 8 if c["apart"] else n)
        for t, n in at.items():
            flat[t] = normal(n, dtype=TYPES[t])
        s["grads"] = [flat[t][a:a + n].view(shape) for t, a, shape, n in places]
        for x in s["grads"]:                # gradients of different layers are of different sizes
            x.mul_(10.0 ** float(-3 * torch.rand((), generator=g, device="cuda")))
        s["flat"] = [torch.zeros_like(flat[t]) for t in sorted(flat)]
        to = dict(zip(sorted(flat), s["flat"]))
        s["out"] = [to[t][a:a + n].view(shape) for t, a, shape, n in places]
        return s
    dt, T, W = TYPES[c["dtype"]], c["tokens"], c["width"]
    if c["absent"]:
        s["pos"] = torch.zeros(T, dtype=torch.int32, device="cuda")
        s["pos"][torch.rand(T, generator=g, device="cuda") < c["absent"]] = -1

    def tokens(*shape, dtype=dt, size=1.0):
        x = (torch.randn(shape, generator=g, device="cuda") * size).to(dtype)
        if s["pos"] is not None:
            x[s["pos"] < 0] = float("nan")
        return x

    if c["op"] in ("norm", "norm_train", "serve"):
        # channels of different sizes, as a residual has them
        s.update(x=tokens(T, W), residual=tokens(T, W, dtype=TYPES[c["stream"]], size=2 * torch.exp(0.5 * normal(W))), weight=1 + 0.2 * normal(W))
    if c["op"] == "norm_train":
        s.update(dy=tokens(T, W), d_total=tokens(T, W, dtype=TYPES[c["stream"]]))
    if c["op"] in ("product", "serve"):
        s["weight8"] = _rows8(normal(c["out"], W) * W ** -0.5)
        s["bias"] = normal(c["out"])
    if c["op"] == "product":
        s["rows8"] = _rows8(normal(T, W) * torch.exp(0.5 * normal(T, 1)))
    if c["op"].startswith("gated"):
        s.update(x=tokens(T, W), w_gate=normal(c["hidden"], W, dtype=dt) * W ** -0.5, w_up=normal(c["hidden"], W, dtype=dt) * W ** -0.5, dh=None)
        if c["op"] == "gated_train":
            s["dh"] = tokens(T, c["hidden"])
    return s


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op.startswith("norm"):
        return _norm_plain(s)
    if op == "clip":
        return _clip_plain(s)
    return _gated_plain(s) if op.startswith("gated") else _product_plain(s)


def _run_own(s):
    import paper_2305_16588_amd as lgp
    c = s["case"]
    if c["op"] == "clip":
        return [lgp.clip_gradients(s["grads"], c["most"], out=s["out"]), *s["flat"]]
    if c["op"].startswith("norm"):
        y, total = lgp.add_norm(s["x"], s["residual"], s["weight"], pos=s["pos"], eps=EPS)
        if c["op"] == "norm":
            return [y, total]
        return [y, total, *lgp.add_norm_backward(s["dy"], s["d_total"], total, s["weight"], pos=s["pos"], eps=EPS)]
    if c["op"].startswith("gated"):
        h = lgp.gated_linear(s["x"], s["w_gate"], s["w_up"], act=c["act"], pos=s["pos"])
        if c["op"] == "gated":
            return [h]
        return [h, *lgp.gated_linear_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], act=c["act"], pos=s["pos"])]
    if "weight" not in s.get("own", ()):          # a program keeps what holds its weights
        s["own"] = dict(weight=lgp.Rows8(*s["weight8"], c["width"]))
    w = s["own"]["weight"]
    if c["op"] == "product":
        return [lgp.linear_rows8(lgp.Rows8(*s["rows8"], c["width"]), w, bias=s["bias"], dtype=TYPES[c["dtype"]])]
    rows, total = lgp.add_norm_rows8(s["x"], s["residual"], s["weight"], pos=s["pos"], eps=EPS)
    return [lgp.linear_rows8(rows, w, bias=s["bias"], dtype=TYPES[c["dtype"]]), total]


def _there(s, x):
    """Rows without a token as zeros, in 32 bits."""
    return x.float() if s["pos"] is None else torch.where((s["pos"] >= 0)[:, None], x.float(), 0.0)


def _normed(s):
    total = (_there(s, s["x"]) + _there(s, s["residual"])).to(s["residual"].dtype)
    t = total.float()
    r = torch.rsqrt(t.square().mean(1, keepdim=True) + EPS)
    return total, t * r, r


def _norm_plain(s):
    total, n, r = _normed(s)
    dt = s["x"].dtype
    y = (n * s["weight"]).to(dt)
    if s["case"]["op"] == "norm":
        return [y, total]
    dy = _there(s, s["dy"])
    dw = (dy * n).sum(0)
    dy = dy * s["weight"]
    d = r * (dy - n * (dy * n).mean(1, keepdim=True)) + s["d_total"].float()
    d = _there(s, d)
    return [y, total, d.to(dt), d.to(total.dtype), dw]


def _product_plain(s):
    c = s["case"]
    (w, w_scale), more = s["weight8"], []
    if c["op"] == "product":
        v, scale = s["rows8"]
        v = v.float()
    else:
        total, n, _ = _normed(s)
        y = n * s["weight"]
        scale = (y.abs().amax(1) / 127).clamp(min=2.0 ** -126)
        v = torch.nn.functional.pad((y / scale[:, None]).round().clamp(-127, 127), (0, -c["width"] % 16))
        more = [total]
    out = (v @ w.float().t()) * scale[:, None] * w_scale + s["bias"]
    return [_there(s, out).to(TYPES[c["dtype"]]), *more]


def _gated_plain(s):
    c, dt = s["case"], s["x"].dtype
    x, wg, wu = _there(s, s["x"]), s["w_gate"].float(), s["w_up"].float()
    g, u = x @ wg.t(), x @ wu.t()
    p = torch.sigmoid(g) if c["act"] == "silu" else 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    a = g * p
    h = (a * u).to(dt)
    if c["op"] == "gated":
        return [h]
    slope = p + a * (1 - p) if c["act"] == "silu" else p + g * torch.exp(-0.5 * g * g) * (0.5 / math.pi) ** 0.5
    dh = _there(s, s["dh"])
    du, dg = dh * a, dh * u * slope
    del g, u, p, a, slope, dh
    return [h, (dg @ wg + du @ wu).to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt)]


def _clip_plain(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    by = (s["case"]["most"] / norm).clamp(max=1.0).float()
    _ = [o.copy_(g.float() * by) for o, g in zip(s["out"], s["grads"])]
    return [norm.float(), *s["flat"]]


def work(case):
    c = case
    if c["op"] == "clip":
        n = {t: sum(math.prod(x) for x, u in _gradients(c) if u == t) for t in SIZE}
        return {"bytes": 2 * sum(n[t] * SIZE[t] for t in n), "flops": 3 * sum(n.values())}
    T, W, has, size = c["tokens"], c["width"], 1 - c["absent"], SIZE[c["dtype"]]
    if c["op"].startswith("norm"):
        stream = SIZE[c["stream"]]
        b, f = T * W * (1 + has) * (size + stream), 6
        if c["op"] == "norm_train":         # the sum, its gradient and the result's again, one gradient written, two where their types differ
            b, f = b + T * W * (has * (size + 2 * stream) + stream + (size if size != stream else 0)), 20
        return {"bytes": b + 4 * W, "flops": T * W * has * f}
    if c["op"] in ("product", "serve"):
        b = W * c["out"] + 8 * c["out"] + T * c["out"] * size
        b += T * W if c["op"] == "product" else T * W * (has * (size + SIZE[c["stream"]]) + SIZE[c["stream"]])
        return {"bytes": b, "flops": 2 * T * has * W * c["out"]}
    b, f = (T * has * W + 2 * c["hidden"] * W + T * c["hidden"]) * size, 4
    if c["op"] == "gated_train":            # x and the weights again, the gradients of all three and of the result
        b, f = b + (T * (has + 1) * W + 4 * c["hidden"] * W + T * has * c["hidden"]) * size, 16
    return {"bytes": b, "flops": f * T * has * W * c["hidden"]}


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "clip":
        return _clip_exact(s, case)
    if op.startswith("norm"):
        return _norm_exact(s, case)
    return _gated_exact(s, case) if op.startswith("gated") else _product_exact(s, case)


def _blocks(s, c, each):
    """Runs of rows, and which of them hold tokens."""
    for lo in range(0, c["tokens"], each):
        at = torch.arange(lo, min(c["tokens"], lo + each), device="cuda")
        yield at if s["pos"] is None else at[s["pos"][at] >= 0]


def _sum_and_norm(s, at):
    total = (s["x"][at].double() + s["residual"][at].double()).to(s["residual"].dtype)        # what is kept of the sum is what is normed
    size = torch.sqrt((total.double() ** 2).sum(1) / total.shape[1] + EPS)[:, None]
    return total, total.double() / size, size


def _norm_exact(s, c):
    T, W, train = c["tokens"], c["width"], c["op"] == "norm_train"
    y, total = (torch.zeros(T, W, dtype=torch.float64, device="cuda") for _ in range(2))
    d, dw = torch.zeros_like(y) if train else None, torch.zeros(W, dtype=torch.float64, device="cuda")
    w = s["weight"].double()
    for at in _blocks(s, c, 1 << 15):
        t, n, size = _sum_and_norm(s, at)
        total[at], y[at] = t.double(), n * w
        if train:
            dy = s["dy"][at].double()
            dw += torch.einsum("tw,tw->w", dy, n)
            along = torch.einsum("tw,tw->t", dy * w, n)[:, None] / W
            d[at] = s["d_total"][at].double() + (dy * w - along * n) / size
    return [y, total, d, d, dw] if train else [y, total]


def _product_exact(s, c):
    T, O, W = c["tokens"], c["out"], c["width"]
    out = torch.zeros(T, O, dtype=torch.float64, device="cuda")
    total = torch.zeros(T, W, dtype=torch.float64, device="cuda") if c["op"] == "serve" else None
    held = (s["weight8"][0][:, :W].double() * s["weight8"][1].double()[:, None]).t().contiguous()
    for at in _blocks(s, c, 1 << 15):
        if c["op"] == "product":
            x = s["rows8"][0][at, :W].double() * s["rows8"][1][at].double()[:, None]
        else:
            t, n, _ = _sum_and_norm(s, at)
            y = n * s["weight"].double()
            step = y.abs().max(1, keepdim=True).values / 127
            x = torch.where(step > 0, torch.round(y / step) * step, 0.0)
            total[at] = t.double()
        out[at] = x @ held + s["bias"].double()
    return [out] if total is None else [out, total]


def _gated_exact(s, c):
    T, W, H, train = c["tokens"], c["width"], c["hidden"], c["op"] == "gated_train"
    f8 = dict(dtype=torch.float64, device="cuda")
    h, dx = torch.zeros(T, H, **f8), torch.zeros(T, W, **f8) if train else None
    dwg, dwu = (torch.zeros(H, W, **f8) if train else None for _ in range(2))
    wg, wu = s["w_gate"].double(), s["w_up"].double()
    for at in _blocks(s, c, 1 << 13):
        x = s["x"][at].double()
        g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        share = 1 / (1 + torch.exp(-g)) if c["act"] == "silu" else 0.5 * torch.erfc(-g / math.sqrt(2))
        h[at] = g * share * u
        if train:
            dh = s["dh"][at].double()
            more = g * share * (1 - share) if c["act"] == "silu" else g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
            du, dg = dh * g * share, dh * u * (share + more)
            dx[at] = torch.mm(dg, wg) + torch.mm(du, wu)
            dwg += torch.mm(dg.t(), x)
            dwu += torch.mm(du.t(), x)
    return [h, dx, dwg, dwu] if train else [h]


def _clip_exact(s, c):
    norm = math.sqrt(math.fsum(float(torch.dot(g.double().flatten(), g.double().flatten())) for g in s["grads"]))
    by = min(1.0, c["most"] / norm)
    flat = [torch.zeros_like(f, dtype=torch.float64) for f in s["flat"]]
    for g, o in zip(s["grads"], s["out"]):
        k = next(i for i, f in enumerate(s["flat"]) if f.dtype == o.dtype)
        a = o.storage_offset()
        flat[k][a:a + o.numel()] = g.double().flatten() * by
    return [torch.tensor(norm, dtype=torch.float64), *flat]
