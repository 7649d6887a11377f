"""What a layer has around its attention at the ends of its range: numbers near the types' ends, sums that are known exactly, places beyond 32 bits, and every form of
the products on streams, in captured graphs and repeated bit by bit."""
import math

import pytest
import torch

import dense_common as ref
from layer_common import check
from test_gpu_9_dense import BF16, F16, F32, draw, lgp, rows_of, slots

pytestmark = pytest.mark.gpu


# ---- the gated pair, where every number along the way is a power of two or a sum of few bits: results are known exactly, and one token in the wrong place shows

# few tokens, small tiles, large tiles, rows that pass by the weights (all four lengths of the sum); gradients by tiles of every size, with parts of the sum
FORMS = [(1, 8, 1), (8, 1000, 130), (40, 72, 300), (9, 264, 129), (300, 64, 80), (1025, 256, 683), (4097, 64, 96), (4000, 136, 1100), (66_003, 40, 100), (65_600, 64, 9), (66_003, 120, 64),
         (66_003, 256, 100), (33_000, 512, 130), (40_010, 1024, 300), (40_010, 1024, 800)]


def powers(shape, low, high, seed):
    """+-2^low ... 2^high, drawn evenly."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    size = torch.randint(low, high + 1, shape, generator=g, device="cuda").double()
    return torch.exp2(size) * (1 - 2 * torch.randint(0, 2, shape, generator=g, device="cuda").double())


def one_hot(tokens, width, dtype, place, size):
    x = torch.zeros(tokens, width, dtype=dtype, device="cuda")
    x[torch.arange(tokens, device="cuda"), place] = size
    return x


def run_known(tokens, width, hidden, dtype, act, size, gate, up, grad, pos=None, share=1.0, seed=1):
    """Token t is `size` at one place.  Gates are +-size 2^gate, at which an activation is its argument or zero and its slope 1 or 0; the other
    projection's results are +-size 2^up and gradients of h +-2^grad, of `share` of the tokens.  Every product and every sum of them is exact in 32 bits."""
    L = lgp()
    place = torch.arange(tokens, device="cuda") * 7 % width
    x, dh = one_hot(tokens, width, dtype, place, size), powers((tokens, hidden), *grad, seed).to(dtype)
    if share < 1:
        dh[torch.rand(tokens, generator=torch.Generator(device="cuda").manual_seed(seed + 3), device="cuda") >= share] = 0
    wg, wu = powers((hidden, width), *gate, seed + 1).to(dtype), powers((hidden, width), *up, seed + 2).to(dtype)
    live = ref.live_rows(tokens, pos, "cuda")[:, None]
    g, u = size * wg.double().t()[place], size * wu.double().t()[place]
    on, d = (g > 0) & live, torch.where(live, dh.double(), 0.0)
    a = torch.where(on, g, 0.0)
    dg, du = torch.where(on, d * u, 0.0), d * a
    X = torch.where(live, x.double(), 0.0)
    want = dict(h=a * u, dx=dg @ wg.double() + du @ wu.double(), dw_gate=dg.t() @ X, dw_up=du.t() @ X)
    if pos is not None:
        x[pos < 0], dh[pos < 0] = math.nan, math.nan
    got = dict(h=L.gated_linear(x, wg, wu, act=act, pos=pos))
    got.update(zip(("dx", "dw_gate", "dw_up"), L.gated_linear_backward(dh, x, wg, wu, act=act, pos=pos)))
    for name, w in want.items():
        # all of them have less than 24 bits: fp32 holds them, and they are rounded once from there
        assert torch.equal(w.float().double(), w), name
        assert torch.isfinite(w.to(dtype)).all(), name
        assert torch.equal(got[name], w.float().to(dtype)), (name, int((got[name] != w.float().to(dtype)).sum()))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens,width,hidden", FORMS)
def test_gated_of_gates_beyond_24_bits(tokens, width, hidden, act):
    """From 2^24 on 1 + g is g or its neighbour, but the activation's slope is 1."""
    run_known(tokens, width, hidden, BF16, act, 2.0 ** 13, gate=(11, 13), up=(-13, -12), grad=(0, 1))
    run_known(tokens, width, hidden, BF16, act, 2.0 ** 13, gate=(11, 13), up=(-13, -12), grad=(0, 1), pos=slots(tokens, 3), seed=7)


@pytest.mark.parametrize("tokens,width,hidden", FORMS)
def test_gated_of_fp16_gradients_far_below_its_smallest(tokens, width, hidden):
    """The gradients of a gate are 2^-26 and 2^-25, neither of which fp16 holds; those of x and the weights it does."""
    for pos in (None, slots(tokens, 3)):
        run_known(tokens, width, hidden, F16, "silu", 8.0, gate=(4, 5), up=(-16, -16), grad=(-13, -12), pos=pos)


@pytest.mark.parametrize("tokens,width,hidden", FORMS)
def test_gated_of_fp16_gradients_beyond_its_largest(tokens, width, hidden):
    """The gradient of a gate is 2^19 half of the time, beyond fp16; those of x and the weights are not.  Gates are zero, where silu's slope is 1/2."""
    L = lgp()
    half = width // 2
    for pos in (None, slots(tokens, 3)):
        live = ref.live_rows(tokens, pos, "cuda")[:, None]
        place = torch.arange(tokens, device="cuda") * 7 % half
        x, dh = one_hot(tokens, width, F16, place, 2.0 ** -9), powers((tokens, hidden), 13, 14, 1).to(F16)
        dh[torch.rand(dh.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") > 1 / 16] = 0
        wg, wu = powers((hidden, width), -10, -9, 3).to(F16), powers((hidden, width), 14, 15, 4).to(F16)
        wg[:, :half] = 0
        dg = torch.where(live, dh.double(), 0.0) * 2.0 ** -9 * wu.double().t()[place] / 2
        want = dict(dx=dg @ wg.double(), dw_gate=dg.t() @ torch.where(live, x.double(), 0.0), dw_up=torch.zeros(hidden, width, dtype=torch.float64, device="cuda"))
        if pos is not None:
            x[pos < 0], dh[pos < 0] = math.nan, math.nan
        for (name, w), got in zip(want.items(), L.gated_linear_backward(dh, x, wg, wu, pos=pos)):
            assert torch.equal(w.float().double(), w) and torch.isfinite(w.half()).all(), name
            assert torch.equal(got, w.half()), name


@pytest.mark.parametrize("tokens", [8, 9, 64, 65, 300, 4097])
def test_gated_of_fp16_keeps_its_error_at_every_size_of_gradients(monkeypatch, tokens):
    """Gradients of h from 2^-20 to 2^12 and a row of zeros: but for results below fp16's smallest, errors are those of roundings by 2^-11.  The gradients of the projections'
    results are lifted by a power of two, B 1.2 to 2^14 or more where B is the largest |dh| |x| of a token times the largest |w|, and fp16 keeps 2^-25: 1.2 2^-39 of B."""
    L = lgp()
    x, wg, wu = draw((tokens, 96), F16, 1, 0.1), draw((200, 96), F16, 2, 0.1), draw((200, 96), F16, 3, 0.1)
    dh = draw((tokens, 200), F16, 4, 0.25)
    dh[3] = 0
    monkeypatch.setitem(ref.TINY, F16, 0.0)
    norm = max(float(w.double().norm(dim=1).max()) for w in (wg, wu))
    for power in (-18, -10, 0, 8):
        d = (dh.double() * 2.0 ** power).half()
        want = ref.gated(x, wg, wu, "silu", None, d)
        low = 2.0 ** -39 * 1.2 * float((d.abs().amax(1).double() * x.double().norm(dim=1)).max()) * norm
        more = dict(dx=low * (wg.double().abs() + wu.double().abs()).sum(0), dw_gate=low * x.double().abs().sum(0), dw_up=low * x.double().abs().sum(0))
        for name, got in zip(("dx", "dw_gate", "dw_up"), L.gated_linear_backward(d, x, wg, wu)):
            val, tol = want[name]
            check(got, (val, tol + more[name] + 2.0 ** -25), (name, power))
    clean = L.gated_linear_backward(dh, x, wg, wu)[0]
    for bad in (math.inf, math.nan):
        d = dh.clone()
        d[5, 7] = bad
        dx, dg, _ = L.gated_linear_backward(d, x, wg, wu)
        odd = torch.arange(tokens, device="cuda") == 5
        assert torch.equal(dx[~odd], clean[~odd]) and not torch.isfinite(dx[5]).any() and not torch.isfinite(dg[7]).any()
        assert torch.isfinite(dg[torch.arange(200, device="cuda") != 7]).all()


# ---- gradients' clipping

def rounded_once(x, dtype):
    """Numbers of 64 bits as the nearest of `dtype`, ties to even, in whole numbers of its last places."""
    bits, low = {F16: (11, -24), BF16: (8, -133), F32: (24, -149)}[dtype]
    step = torch.exp2((torch.frexp(x.abs())[1] - bits).clamp(min=low).double())
    return torch.round(x / step) * step


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_clipped_gradients_are_rounded_once(dtype):
    """Every positive number of the type below 2^14 (fp32: many), by factors that are known exactly: the norm is a power of two, which one gradient has almost alone."""
    L = lgp()
    if dtype is F32:
        g = torch.rand(200_000, generator=torch.Generator().manual_seed(1)).cuda()
    else:
        g = torch.arange(1, 1 << 15).to(torch.int16).view(dtype)
        g = g[torch.isfinite(g) & (g < 2.0 ** 14)].cuda()
    whole = 2.0 ** 60                            # beside it all other squares, below 2^28 each and 2^43 together, are less than half of a place of 2^120
    first = torch.full((1,), whole, device="cuda")
    off = 0
    for i in range(40):
        most = whole * (1 - math.ldexp(1 + 977 * i, -17))          # the factor has 17 bits, so products with numbers of 24 are exact in 64
        out = [torch.empty_like(first), torch.empty_like(g)]
        assert float(L.clip_gradients([first, g], most, out=out)) == whole and float(out[0]) == most
        want = rounded_once(g.double() * (most / whole), dtype)
        off += int((out[1].double() != want).sum())
    assert off == 0


# ---- the norm

def run_far(tokens, width, dtype, stream, size, eps, pos=None, g_size=1.0, seed=1, back=True):
    """Rows of numbers around `size`, their norm and gradients, within the bounds of other rows."""
    L = lgp()
    res = (draw((tokens, width), F32, seed).double() * size).to(stream)
    x, w = torch.zeros(tokens, width, dtype=dtype, device="cuda"), 1 + draw((width,), F32, seed + 1, 0.3)
    dy = (draw((tokens, width), F32, seed + 2).double() * g_size).to(dtype)
    if pos is not None:
        res[pos < 0] = math.nan
    assert torch.isfinite(res[ref.live_rows(tokens, pos, "cuda")]).all()
    y, total = L.add_norm(x, res, w, pos=pos, eps=eps)
    want = ref.add_norm(x, res, w, pos, eps)
    check(y, want["y"], "y")
    if back:
        exact = ref.add_norm(None, None, w, pos, eps, dy, None, total)
        for got, name in zip(L.add_norm_backward(dy, None, total, w, pos=pos, eps=eps), ("dx", "d_residual", "dw")):
            val, tol = exact[name]
            check(got, (val, tol + 2.0 ** -134), name)          # the smallest numbers lose digits
    rows, _ = L.add_norm_rows8(x, res, w, pos=pos, eps=eps)
    ref.rows8(*want["y32"], rows.values, rows.scales, ref.live_rows(tokens, pos, "cuda"))


@pytest.mark.parametrize("width", [3, 33, 256, 1000, 2500, 9000])
@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F32)])
def test_norm_of_rows_whose_squares_32_bits_do_not_hold(width, dtype, stream):
    """Sums of squares beyond 2^128 or below 2^-126; with an eps that matters beside them and without."""
    for size in (2.0 ** 63, 2.0 ** 80, 2.0 ** 118):
        for eps in (1e-6, 0.0):
            run_far(21, width, dtype, stream, size, eps, g_size=1.0 if dtype is F16 else 2.0 ** 20, pos=slots(21, width))
    for size in (2.0 ** -50, 2.0 ** -64, 2.0 ** -80, 2.0 ** -110):
        for eps in (1e-6, size * size if size > 2.0 ** -63 else 0.0, 0.0):
            run_far(21, width, dtype, stream, size, eps, g_size=2.0 ** -30, pos=slots(21, width), back=dtype is not F16)       # fp16 does not hold such gradients


def test_gradients_of_a_norm_that_is_not_finite_are_not():
    """A NaN spoils its row's gradients and all of the weight's, an infinity its own element's; zeros with an eps of zero have no norm."""
    L = lgp()
    for width in (40, 300, 3000):
        total, dy, w = draw((50, width), F32, 1), draw((50, width), F32, 2), 1 + draw((width,), F32, 3, 0.1)
        clean, _, _ = L.add_norm_backward(dy, None, total, w)
        odd, place = torch.arange(50, device="cuda") == 7, torch.arange(width, device="cuda") == 3
        total[7, 3] = math.nan
        dx, _, dw = L.add_norm_backward(dy, None, total, w)
        assert torch.isnan(dx[7]).all() and torch.isnan(dw).all() and torch.equal(dx[~odd], clean[~odd])
        total[7, 3] = math.inf
        dx, _, dw = L.add_norm_backward(dy, None, total, w)
        assert torch.isnan(dw[3]) and torch.isfinite(dw[~place]).all() and torch.equal(dx[~odd], clean[~odd])
        total[7] = 0
        dx, _, dw = L.add_norm_backward(dy, None, total, w, eps=0.0)
        assert torch.isnan(dx[7]).all() and torch.isnan(dw).all()
        y, _ = L.add_norm(total, None, w, eps=0.0)
        assert torch.isnan(y[7]).all() and torch.isfinite(y[~odd]).all()


# ---- every form on streams, in captured graphs and repeated bit by bit

def all_forms():
    """(calls, inputs): the gated pair and its gradients with lists and without, by rows that pass and by tiles of every size, and the products in 8 bits by every form."""
    L = lgp()
    calls, inputs = [], []
    for tokens, width, hidden, dtype, listed in ((30, 64, 48, BF16, False), (700, 256, 130, F16, True), (5000, 128, 96, F16, True), (4500, 256, 683, BF16, True), (66_003, 64, 40, F16, False),
                                                 (70_001, 128, 40, BF16, True), (66_003, 250 // 8 * 8, 100, F16, True), (33_000, 512, 130, BF16, True), (4000, 136, 1100, F16, False),
                                                 (9000, 520, 700, BF16, True)):
        x, dh = draw((tokens, width), dtype, tokens), draw((tokens, hidden), dtype, tokens + 1, 0.1)
        wg, wu = draw((hidden, width), dtype, tokens + 2, width ** -0.5), draw((hidden, width), dtype, tokens + 3, width ** -0.5)
        pos = slots(tokens, tokens) if listed else None
        calls.append(lambda stream=None, a=(x, wg, wu), p=pos: [L.gated_linear(*a, pos=p, stream=stream)])
        calls.append(lambda stream=None, d=dh, a=(x, wg, wu), p=pos: list(L.gated_linear_backward(d, *a, pos=p, stream=stream)))
        inputs += [x, dh]
    for tokens, width, channels in ((20, 1000, 300), (276, 256, 768), (70_001, 100, 130), (70_001, 256, 130), (70_001, 500, 130), (70_001, 1000, 130), (33_001, 1040, 300)):
        x, weight, bias = draw((tokens, width), F16, tokens + width), rows_of(channels, width, tokens + 1), draw((channels,), F32, tokens + 2)
        pos = slots(tokens, width)
        calls.append(lambda stream=None, x=x, w=weight, b=bias, p=pos: [L.linear_rows8(L.pack_rows(x, pos=p, stream=stream), w, bias=b, dtype=F32, stream=stream)])
        inputs.append(x)
    return calls, inputs


def run_all(calls, stream=None):
    return [t for call in calls for t in call(stream)]


def alike(got, want):
    assert len(got) == len(want)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def test_all_forms_are_the_same_bit_by_bit_and_on_another_stream():
    calls, _ = all_forms()
    first = run_all(calls)
    assert all(torch.isfinite(t).all() for t in first)
    alike(run_all(calls), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run_all(calls, side)
    torch.cuda.current_stream().wait_stream(side)
    alike(got, first)


def test_all_forms_captured_and_replayed():
    calls, inputs = all_forms()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run_all(calls)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run_all(calls)
    for seed in range(3):
        for t in inputs:
            t.copy_(draw(t.shape, t.dtype, 100 + seed, 0.5 ** seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        alike(got, run_all(calls))


# ---- places beyond 32 bits

def few_rows(tokens):
    return torch.tensor([0, 1, 255, tokens // 2 + 3, tokens - 300, tokens - 1], device="cuda")


def check_far(tokens, width, hidden, dtype, pos=None, x=None):
    """All rows are zeros but for a few, whose results stand where they belong; all others are zeros."""
    L = lgp()
    at = few_rows(tokens)
    if x is None:
        x = torch.zeros(tokens, width, dtype=dtype, device="cuda")
    dh = torch.zeros(tokens, hidden, dtype=dtype, device="cuda")
    x[at], dh[at] = draw((len(at), width), dtype, 1), draw((len(at), hidden), dtype, 2)
    wg, wu = draw((hidden, width), dtype, 3, width ** -0.5), draw((hidden, width), dtype, 4, width ** -0.5)
    if pos is not None:
        pos[at] = 1
    want = ref.gated(x[at], wg, wu, "silu", None, dh[at])
    h = L.gated_linear(x, wg, wu, pos=pos)
    check(h[at], want["h"], "h")
    h[at] = 0
    assert not h.any()
    del h
    dx, dg, du = L.gated_linear_backward(dh, x, wg, wu, pos=pos)
    check(dx[at], want["dx"], "dx")
    dx[at] = 0
    assert not dx.any()
    check(dg, want["dw_gate"], "dw_gate")
    check(du, want["dw_up"], "dw_up")


def test_gated_beyond_32_bits():
    """Elements of h, of its gradient and of x whose places pass 2^31, bytes beyond 2^32; the projections' gradients, two for each element of h, pass 2^32."""
    check_far(300_000, 520, 7400, BF16)               # large tiles
    check_far((1 << 24) - 5, 136, 40, F16)            # rows of x
    check_far((1 << 24) - 5, 64, 136, BF16)           # rows that pass by the weights


def test_gated_with_lists_beyond_32_bits():
    pos = torch.full(((1 << 24) - 5,), -1, dtype=torch.int32, device="cuda")
    pos[::3] = 0
    check_far((1 << 24) - 5, 64, 136, F16, pos=pos)
    # rows of x so far apart that units of 16 bytes come near 2^32, and further, where there is no list
    for tokens, listed in ((8190, 1), (8300, 0)):
        row = (1 << 22) - 8
        assert (tokens * row < 1 << 35) == listed
        x = torch.empty(tokens * row, dtype=BF16, device="cuda").as_strided((tokens, 64), (row, 1))
        x.zero_()
        pos = torch.zeros(tokens, dtype=torch.int32, device="cuda")
        pos[1::2] = -1
        for hidden in (96, 600, 2100):
            check_far(tokens, 64, hidden, BF16, pos=pos, x=x)
        del x


@pytest.mark.parametrize("tokens,width,channels", [((1 << 24) - 5, 64, 136), ((1 << 24) - 5, 1040, 136), (600_000, 300, 4000), (200, 40, (1 << 24) - 5)])
def test_products_in_8_bits_beyond_32_bits(tokens, width, channels):
    """Results whose places pass 2^31 (and bytes of rows 2^32)."""
    L = lgp()
    weight, rows = rows_of(channels, width, 1), rows_of(tokens, width, 2)
    out = L.linear_rows8(rows, weight, dtype=BF16)
    for at in (slice(0, 300), slice(tokens // 2, tokens // 2 + 100), slice(tokens - 300, None)):
        v, s = rows.values[at].float(), rows.scales[at].double()
        for c in (slice(0, 200), slice(max(0, channels - 200), None)):
            want = (v @ weight.values[c].float().t()).double() * weight.scales[c].double() * s[:, None]        # sums of 1040 products below 2^14: exact in fp32
            check(out[at, c], (want, 2.0 ** -22 * want.abs() + 2.0 ** -8 * want.abs()))


# ---- weights' gradients of large batches

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tokens,width,hidden", FORMS)
def test_gated_of_sums_that_are_exact(tokens, width, hidden, act, dtype):
    """A token that is left out, read twice or put elsewhere changes a whole number."""
    for pos in (None, slots(tokens, 3)):
        run_known(tokens, width, hidden, dtype, act, 8.0, gate=(4, 5), up=(-3, -2), grad=(-6, -5), pos=pos)
    run_known(tokens, width, hidden, dtype, act, 8.0, gate=(4, 5), up=(-3, -2), grad=(-6, -5), share=min(1.0, 300 / tokens))
    pos = slots(tokens, 3)
    pos[:tokens // 3] = -1
    pos[-tokens // 5:] = -1
    run_known(tokens, width, hidden, dtype, act, 8.0, gate=(4, 5), up=(-3, -2), grad=(-6, -5), pos=pos)
