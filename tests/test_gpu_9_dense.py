"""What a layer has around its attention, against its definitions in 64 bits (tests/dense_common.py), at the sizes, masks and layouts where it can go
wrong; streams, captured graphs and runs that are repeated bit by bit."""
import math

import pytest
import torch

import dense_common as ref
from layer_common import UNIT, check

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)]


def lgp():
    import paper_2305_16588_amd
    return paper_2305_16588_amd


def draw(shape, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * size).to(dtype)


def slots(tokens, seed, share=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.where(torch.rand(tokens, generator=g, device="cuda") < share, -1, torch.arange(tokens, device="cuda")).to(torch.int32)


def strided(t, more=3):
    """The same rows further apart, at an odd place."""
    wide = torch.full((t.shape[0], t.shape[1] + more), math.nan, dtype=t.dtype, device=t.device)
    wide[:, 1:1 + t.shape[1]] = t
    return wide[:, 1:1 + t.shape[1]]


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=7.0), torch.nan_to_num(b.float(), nan=7.0))


def run_norm(tokens, width, dtype, stream, pos=None, seed=1, adds=True, apart=False, eps=1e-6, later=True):
    L = lgp()
    x, w = draw((tokens, width), dtype, seed), 1 + draw((width,), F32, seed + 1, 0.3)
    res = draw((tokens, width), stream, seed + 2, 2.0) if adds else None
    dy, dt = draw((tokens, width), dtype, seed + 3), draw((tokens, width), stream, seed + 4) if later else None
    if pos is not None:
        for t in (x, res, dy, dt):
            if t is not None:
                t[pos < 0] = math.nan
    if apart:
        x, res = strided(x), res if res is None else strided(res, 8)
    y, total = L.add_norm(x, res, w, pos=pos, eps=eps)
    want = ref.add_norm(x, res, w, pos, eps)
    if adds:
        assert total.dtype is stream and same(total, want["total"])
    else:
        assert total is x
    check(y, want["y"], "y")
    back = ref.add_norm(None, None, w, pos, eps, dy, dt, total)
    dx, dr, dw = L.add_norm_backward(dy, dt, total, w, pos=pos, eps=eps)
    assert dx.dtype is dtype and dr.dtype is total.dtype
    check(dx, back["dx"], "dx")
    check(dr, back["d_residual"], "d_residual")
    check(dw, back["dw"], "d_weight")
    rows, total8 = L.add_norm_rows8(x, res, w, pos=pos, eps=eps)
    assert same(total8, total)
    ref.rows8(*want["y32"], rows.values, rows.scales, ref.live_rows(tokens, pos, "cuda"))


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("width", [1, 7, 8, 31, 32, 33, 100, 128, 129, 256, 257, 500, 512, 1000, 1024, 1025, 2048, 2049, 4096, 4100, 8192, 8193, 16384])
def test_norm_of_every_width(width, dtype, stream):
    for tokens in (1, 37):
        run_norm(tokens, width, dtype, stream)
    run_norm(70, width, dtype, stream, pos=slots(70, width), apart=True)


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("tokens,width", [(5000, 256), (20_011, 40), (3001, 1024), (1500, 3000)])
def test_norm_of_many_rows(tokens, width, dtype, stream):
    run_norm(tokens, width, dtype, stream, pos=slots(tokens, 3))
    run_norm(tokens, width, dtype, stream, later=False, eps=1e-3)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_norm_without_a_residual(dtype):
    run_norm(300, 250, dtype, dtype, adds=False, pos=slots(300, 5))
    run_norm(1, 4500, dtype, dtype, adds=False)


def test_norm_of_nothing_and_of_zeros():
    L = lgp()
    w = torch.ones(40, device="cuda")
    for n in (0, 1):
        x = torch.zeros(n, 40, dtype=F16, device="cuda")
        y, total = L.add_norm(x, x, w)
        dx, dr, dw = L.add_norm_backward(x, x, total, w)
        rows, _ = L.add_norm_rows8(x, x, w)
        assert all(t.shape == (n, 40) and (t == 0).all() for t in (y, total, dx, dr)) and (dw == 0).all() and rows.shape == (n, 40) and (rows.values == 0).all()
    pos = torch.full((9,), -1, dtype=torch.int32, device="cuda")          # no token at all, and an eps of zero
    x = torch.full((9, 40), math.nan, device="cuda")
    y, total = L.add_norm(x, x, w, pos=pos, eps=0.0)
    dx, _, dw = L.add_norm_backward(x, x, total, w, pos=pos, eps=0.0)
    assert (y == 0).all() and (total == 0).all() and (dx == 0).all() and (dw == 0).all()


def test_norm_keeps_what_is_not_finite_in_its_row():
    L = lgp()
    x, res, w = draw((50, 130), BF16, 1), draw((50, 130), BF16, 2), 1 + draw((130,), F32, 3, 0.1)
    clean, _ = L.add_norm(x, res, w)
    clean8, _ = L.add_norm_rows8(x, res, w)
    x[7, 3], x[9, 129], x[11, 0] = math.nan, math.inf, -math.inf
    y, _ = L.add_norm(x, res, w)
    rows, _ = L.add_norm_rows8(x, res, w)
    odd = torch.zeros(50, dtype=torch.bool, device="cuda")
    odd[[7, 9, 11]] = True
    assert torch.equal(y[~odd], clean[~odd]) and torch.isnan(y[7]).all() and torch.isnan(y[9, 129]) and (y[9, :129] == 0).all()
    assert torch.isnan(rows.scales[odd]).all() and (rows.values[odd] == 0).all()
    assert torch.equal(rows.values[~odd], clean8.values[~odd]) and torch.equal(rows.scales[~odd], clean8.scales[~odd])


def test_rows_of_broadcast_and_same_inputs():
    """One row for all tokens, and the branch as its own residual."""
    L = lgp()
    one, res, w = draw((1, 96), F16, 1), draw((33, 96), F16, 2), 1 + draw((96,), F32, 3, 0.1)
    x = one.expand(33, 96)
    y, total = L.add_norm(x, res, w)
    assert same(total, x.contiguous() + res)
    check(y, ref.add_norm(x, res, w, None, 1e-6)["y"])
    y, total = L.add_norm(res, res, w)
    assert same(total, res + res)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("width", [1, 15, 16, 17, 100, 1000, 5000, 16384])
def test_rows_in_8_bits(width, dtype):
    L = lgp()
    x = draw((50, width), dtype, width) * torch.exp2(torch.randint(-12, 8, (50, 1), generator=torch.Generator().manual_seed(1)).float()).cuda().to(dtype)
    x[3] = 0
    pos = slots(50, 2)
    x[pos < 0] = math.nan
    for t in (x, strided(x)):
        rows = L.pack_rows(t, pos=pos)
        ref.rows8(x.double(), torch.zeros_like(x, dtype=torch.float64), rows.values, rows.scales, pos >= 0)
    assert L.pack_rows(x[:0]).shape == (0, width)


def test_rows_in_8_bits_of_the_smallest_and_largest_numbers():
    L = lgp()
    x = torch.tensor([[1e-45, -1e-45, 0.0], [3e-38, 1e-38, -3e-38], [3e38, -3.4e38, 1.0], [math.inf, 1, 2], [1, math.nan, 2], [2e-36, -1e-36, 0]], device="cuda")
    rows = L.pack_rows(x)
    ref.rows8(x.double(), torch.zeros_like(x, dtype=torch.float64), rows.values, rows.scales, torch.ones(6, dtype=torch.bool, device="cuda"))
    assert torch.isfinite(rows.scales[[0, 1, 2, 5]]).all()


def test_norm_with_autograd():
    L = lgp()
    x, res, w = draw((60, 100), F32, 1).requires_grad_(), draw((60, 100), F32, 2).requires_grad_(), (1 + draw((100,), F32, 3, 0.2)).requires_grad_()
    a, b = draw((60, 100), F32, 4), draw((60, 100), F32, 5)

    def grads(f):
        return torch.autograd.grad(f, (x, res, w))

    y, total = L.add_norm(x, res, w)
    got = grads((y * a).sum() + (total * b).sum())
    t = (x + res).double()
    n = t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6)
    want = torch.autograd.grad(((n * w) * a).sum() + (t * b).sum(), (x, res, w), retain_graph=True)
    for g, v in zip(got, want):
        assert torch.allclose(g, v, rtol=2e-5, atol=1e-5)
    y, total = L.add_norm(x, res, w)                 # one of the results alone
    want = grads(((n * w) * a).sum())
    for g, v in zip(grads((y * a).sum()), want):
        assert torch.allclose(g, v, rtol=2e-5, atol=1e-5)
    y, total = L.add_norm(x, res, w)
    g = torch.autograd.grad((total * b).sum(), (x, res, w), allow_unused=True)
    assert torch.equal(g[0], b) and torch.equal(g[1], b) and (g[2] == 0).all()
    y, total = L.add_norm(x, None, w)
    assert total is x
    gx, gw = torch.autograd.grad((y * a).sum() + (total * b).sum(), (x, w))
    t = x.double()
    wx, ww = torch.autograd.grad((t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6) * w * a).sum() + (t * b).sum(), (x, w))
    assert torch.allclose(gx, wx, rtol=2e-5, atol=1e-5) and torch.allclose(gw, ww, rtol=2e-5, atol=1e-5)
    leaf, other = draw((4, 100), F32, 6).requires_grad_(), draw((4, 100), F32, 7).requires_grad_()
    for _ in range(2):                                # the gradients of both are one tensor, and add up apart
        L.add_norm(leaf, other, w)[1].sum().backward()
    leaf.grad.mul_(5)
    assert (other.grad == 2).all() and (leaf.grad == 10).all()


def test_norm_beyond_32_bits():
    """Elements whose place passes 2^31, and bytes 2^32."""
    L = lgp()
    tokens, width = 4_300_000, 512
    x = torch.zeros(tokens, width, dtype=BF16, device="cuda")
    w = torch.ones(width, device="cuda")
    tail = draw((5, width), BF16, 1)
    x[-5:] = tail
    y, total = L.add_norm(x, x, w)
    assert same(total[-5:], tail + tail)
    check(y[-5:], ref.add_norm(tail, tail, w, None, 1e-6)["y"])
    dx, _, dw = L.add_norm_backward(y, None, total, w)
    check(dx[-5:], ref.add_norm(None, None, w, None, 1e-6, y[-5:], None, total[-5:])["dx"])
    rows, _ = L.add_norm_rows8(x, x, w)
    assert (rows.values[-5:].abs().amax(1) == 127).all() and (rows.values[-1000:-5] == 0).all()


# ---- products in 8 bits

def rows_of(tokens, width, seed, pos=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.zeros(tokens, (width + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    v[:, :width] = torch.randint(-127, 128, (tokens, width), generator=g, device="cuda", dtype=torch.int8)
    s = torch.rand(tokens, generator=g, device="cuda") * 0.1 + 0.001
    if pos is not None:
        s[pos < 0] = math.nan
    return lgp().Rows8(v, s, width, pos=pos)


def run_product(tokens, width, channels, dtype, bias=True, pos=None, seed=1):
    rows, weight = rows_of(tokens, width, seed, pos), rows_of(channels, width, seed + 1)
    b = draw((channels,), F32, seed + 2, 30.0) if bias else None
    out = lgp().linear_rows8(rows, weight, bias=b, dtype=dtype)
    assert out.dtype is dtype
    v = (rows.values.double() @ weight.values.double().T) * weight.scales.double() * rows.scales.double()[:, None]
    want = v + (b.double() if bias else 0.0)
    tol = 4 * 2.0 ** -24 * (v.abs() + want.abs()) + UNIT[dtype] * want.abs() + ref.TINY[dtype]       # the sum's rounding, two products and the addition
    if pos is not None:
        want, tol = torch.where((pos < 0)[:, None], 0.0, want), torch.where((pos < 0)[:, None], 0.0, tol)
    if dtype is F16:                                    # what is too large for the type
        over = want.abs() >= 65520
        want, tol = torch.where(over, torch.sign(want) * math.inf, want), torch.where(over, 0.0, tol)
    check(out, (want, tol))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("tokens,width,channels", [(1, 1, 1), (1, 16, 16), (1, 1024, 1000), (2, 17, 33), (15, 100, 15), (16, 63, 64), (17, 64, 65), (32, 4097, 40), (33, 65, 31),
                                                   (64, 128, 64), (65, 1000, 129), (276, 256, 768), (1000, 250, 300), (1024, 100, 47), (1025, 1008, 257), (3000, 40, 500),
                                                   (40, 20_000, 40), (1100, 9000, 270), (5000, 256, 300), (2000, 500, 130), (1500, 128, 64), (9000, 33, 70), (2000, 1000, 130), (1100, 600, 70)])
def test_products_in_8_bits(tokens, width, channels, dtype):
    run_product(tokens, width, channels, dtype)
    run_product(tokens, width, channels, dtype, bias=False, pos=slots(tokens, 3), seed=7)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("tokens,width,channels", [(66_003, 100, 130), (66_003, 128, 200), (66_003, 250, 130), (40_000, 256, 260), (66_003, 500, 130), (66_003, 1000, 130), (66_003, 1040, 130),
                                                   (33_001, 17, 300)])
def test_products_in_8_bits_of_batches(tokens, width, channels, dtype):
    run_product(tokens, width, channels, dtype)
    run_product(tokens, width, channels, dtype, bias=False, pos=slots(tokens, 3), seed=7)


def test_products_in_8_bits_of_the_largest_sums():
    """Every product 127^2, as wide as rows may be: the sum is just below 2^31."""
    L = lgp()
    for tokens in (1, 40, 1030):
        v = torch.full((tokens, 1 << 17), 127, dtype=torch.int8, device="cuda")
        w = torch.full((40, 1 << 17), -127, dtype=torch.int8, device="cuda")
        out = L.linear_rows8(L.Rows8(v, torch.ones(tokens, device="cuda"), 1 << 17), L.Rows8(w, torch.ones(40, device="cuda"), 1 << 17), dtype=F32)
        assert (out == -float(127 * 127 << 17)).all()


def test_products_in_8_bits_of_nothing_and_of_rows_that_are_not_finite():
    L = lgp()
    w = rows_of(50, 40, 1)
    assert L.linear_rows8(rows_of(0, 40, 2), w).shape == (0, 50)
    for tokens in (6, 60, 1100):
        x = draw((tokens, 40), F32, 3)
        clean = L.linear_rows8(L.pack_rows(x), w)
        x[4, 7] = math.inf
        out = L.linear_rows8(L.pack_rows(x), w)
        odd = torch.arange(tokens, device="cuda") == 4
        assert torch.isnan(out[4]).all() and torch.equal(out[~odd], clean[~odd])


def test_from_the_residual_to_a_product():
    """As a served layer goes: the residual's addition, the norm in 8 bits, the product with a packed weight; within what 8 bits lose."""
    L = lgp()
    x, res, w = draw((300, 250), BF16, 1), draw((300, 250), BF16, 2), 1 + draw((250,), F32, 3, 0.2)
    weight, pos = draw((90, 250), F32, 4, 250 ** -0.5), slots(300, 5)
    x[pos < 0] = math.nan
    packed = L.pack_rows(weight)
    rows, total = L.add_norm_rows8(x, res, w, pos=pos)
    out = L.linear_rows8(rows, packed, dtype=F32)
    y = ref.add_norm(x, res, w, pos, 1e-6)["y32"][0]
    held = packed.values[:, :250].double() * packed.scales.double()[:, None]
    want = y @ held.T
    # half a step of each value, and what 32 bits add to it and to the product
    tol = torch.nan_to_num(rows.scales.double())[:, None] * (0.5 + 2.0 ** -10) * held.abs().sum(1) + 2.0 ** -20 * y.abs() @ held.abs().T
    check(out, (want, tol))
    assert (out[pos < 0] == 0).all()


# ---- the gated pair

def run_gated(tokens, width, hidden, dtype, act, pos=None, seed=1, apart=0, train=True, size=1.0):
    L = lgp()
    x, dh = draw((tokens, width), dtype, seed, size), draw((tokens, hidden), dtype, seed + 1)
    wg, wu = draw((hidden, width), dtype, seed + 2, width ** -0.5), draw((hidden, width), dtype, seed + 3, width ** -0.5)
    if pos is not None:
        x[pos < 0] = math.nan
        dh[pos < 0] = math.nan
    if apart:
        wide = torch.full((tokens, width + apart), math.nan, dtype=dtype, device="cuda")
        wide[:, 8:8 + width] = x
        x = wide[:, 8:8 + width]
    want = ref.gated(x, wg, wu, act, pos, dh if train else None)
    check(L.gated_linear(x, wg, wu, act=act, pos=pos), want["h"], "h")
    if train:
        for got, name in zip(L.gated_linear_backward(dh, x, wg, wu, act=act, pos=pos), ("dx", "dw_gate", "dw_up")):
            check(got, want[name], name)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens,width,hidden", [(1, 8, 1), (1, 64, 64), (2, 72, 65), (5, 264, 300), (8, 1000, 130), (9, 264, 129), (64, 72, 256), (64, 72, 257), (12, 256, 2000), (15, 256, 100), (16, 1000, 33), (17, 64, 130), (33, 40, 683), (64, 128, 128), (100, 8, 7),
                                                 (129, 136, 129), (276, 256, 352), (300, 520, 257), (1000, 96, 500), (1025, 256, 683), (1500, 72, 40), (2500, 264, 300), (4097, 64, 96), (5000, 256, 130),
                                                 (6000, 120, 683), (4500, 320, 90)])
def test_gated_of_every_size(tokens, width, hidden, dtype, act):
    run_gated(tokens, width, hidden, dtype, act)
    run_gated(tokens, width, hidden, dtype, act, pos=slots(tokens, 9), apart=24, seed=5)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_gated_of_many_tokens_and_of_wide_rows(dtype):
    run_gated(20_001, 128, 200, dtype, "silu", pos=slots(20_001, 2))
    run_gated(2100, 2048, 1100, dtype, "gelu")
    run_gated(40, 4096, 2000, dtype, "silu")
    run_gated(3, 24, 9000, dtype, "silu")


@pytest.mark.parametrize("dtype,act", [(F16, "gelu"), (BF16, "silu")])
@pytest.mark.parametrize("tokens,width,hidden", [(66_003, 40, 100), (65_600, 64, 9), (66_003, 120, 64), (65_540, 128, 33), (66_003, 256, 100), (40_000, 200, 300), (66_003, 320, 70), (66_020, 264, 60),
                                                 (33_000, 512, 130), (66_003, 512, 352), (4000, 136, 1100), (40_010, 1024, 800)])
def test_gated_of_batches(tokens, width, hidden, dtype, act):
    """Rows that pass by the weights, and large tiles; rows without a token at the ends, in runs and among others."""
    run_gated(tokens, width, hidden, dtype, act)
    pos = slots(tokens, 3)
    pos[:700] = -1
    pos[tokens // 2:tokens // 2 + 3000] = -1
    pos[-70:] = -1
    run_gated(tokens, width, hidden, dtype, act, pos=pos, apart=8)


def test_gated_of_batches_of_few_tokens():
    """Many rows, of which hardly any have a token."""
    L = lgp()
    for width, hidden in ((256, 64), (1024, 1100)):
        for n in (0, 1, 65):
            pos = torch.full((70_000,), -1, dtype=torch.int32, device="cuda")
            pos[torch.arange(n, device="cuda") * 1000 + 37] = 1
            run_gated(70_000, width, hidden, BF16, "silu", pos=pos)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_gated_of_large_arguments(dtype, act):
    """Gates from the far ends of the activation's range."""
    run_gated(300, 64, 80, dtype, act, size=6.0, train=dtype is BF16)


def test_gated_of_nothing():
    L = lgp()
    w = draw((40, 64), BF16, 1)
    x = torch.empty((0, 64), dtype=BF16, device="cuda")
    assert L.gated_linear(x, w, w).shape == (0, 40)
    dx, dg, du = L.gated_linear_backward(torch.empty((0, 40), dtype=BF16, device="cuda"), x, w, w)
    assert dx.shape == (0, 64) and (dg == 0).all() and (du == 0).all()
    for tokens in (1, 50, 2000):                     # no token at all
        x, pos = torch.full((tokens, 64), math.nan, dtype=BF16, device="cuda"), torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
        dh = torch.full((tokens, 40), math.nan, dtype=BF16, device="cuda")
        assert (L.gated_linear(x, w, w, pos=pos) == 0).all()
        assert all((t == 0).all() for t in L.gated_linear_backward(dh, x, w, w, pos=pos))


def test_gated_keeps_what_is_not_finite_in_its_row():
    L = lgp()
    for tokens in (9, 700, 1500):
        x, wg, wu, dh = draw((tokens, 72), BF16, 1), draw((90, 72), BF16, 2, 0.1), draw((90, 72), BF16, 3, 0.1), draw((tokens, 90), BF16, 4)
        clean, back = L.gated_linear(x, wg, wu), L.gated_linear_backward(dh, x, wg, wu)
        x[5, 3] = math.nan
        h, (dx, _, _) = L.gated_linear(x, wg, wu), L.gated_linear_backward(dh, x, wg, wu)
        odd = torch.arange(tokens, device="cuda") == 5
        assert torch.isnan(h[5]).all() and torch.equal(h[~odd], clean[~odd]) and torch.isnan(dx[5]).all() and torch.equal(dx[~odd], back[0][~odd])


def test_gated_with_autograd():
    L = lgp()
    x, wg, wu, dh = draw((70, 64), BF16, 1).requires_grad_(), draw((96, 64), BF16, 2, 0.1).requires_grad_(), draw((96, 64), BF16, 3, 0.1).requires_grad_(), draw((70, 96), BF16, 4)
    got = torch.autograd.grad(L.gated_linear(x, wg, wu, act="gelu"), (x, wg, wu), dh)
    want = ref.gated(x.detach(), wg.detach(), wu.detach(), "gelu", None, dh)
    for g, name in zip(got, ("dx", "dw_gate", "dw_up")):
        check(g, want[name], name)
    one = draw((1, 64), BF16, 5).requires_grad_()      # a row for all tokens: its gradients add up
    (g,) = torch.autograd.grad(L.gated_linear(one.expand(70, 64), wg.detach(), wu.detach()), one, dh)
    val, tol = ref.gated(one.detach().expand(70, 64), wg.detach(), wu.detach(), "silu", None, dh)["dx"]
    check(g, (val.sum(0, keepdim=True), tol.sum(0, keepdim=True) + 70 * UNIT[BF16] * val.abs().sum(0, keepdim=True)))


# ---- gradients' norm and clipping

def gradients(shapes, seed=1, flat=False):
    out = [draw(shape, dtype, seed + i, 10.0 ** -(i % 4)) for i, (shape, dtype) in enumerate(shapes)]
    if flat:           # end to end in a bucket of each type
        for dtype in (F32, F16, BF16):
            of = [i for i, g in enumerate(out) if g.dtype is dtype]
            bucket = torch.cat([torch.zeros(1, dtype=dtype, device="cuda"), *(out[i].flatten() for i in of)])
            at = 1
            for i in of:
                n = out[i].numel()
                out[i] = bucket[at:at + n].view(out[i].shape)
                at += n
    return out


MANY = [((7,), F32), ((300, 70), BF16), ((0,), F16), ((1,), BF16), ((129, 129), F16), ((), F32), ((40_000,), BF16), ((16_384,), F32), ((16_385,), F16), ((5, 0), F32)]


def check_clip(grads, most, stays):
    L = lgp()
    norm, want = ref.clip(grads, most)
    given = [g.clone() for g in grads]
    out = None if stays else [torch.full_like(g, 7.0) for g in grads]
    got = L.clip_gradients(grads, most, out=out)
    assert got.shape == () and got.dtype is F32 and abs(float(got) - norm) <= 2.0 ** -23 * norm
    assert abs(float(L.gradient_norm(given)) - norm) <= 2.0 ** -23 * norm
    for g, o, w in zip(given, grads if stays else out, want):
        tiny = {F32: 2.0 ** -150, F16: 2.0 ** -25, BF16: 2.0 ** -134}[g.dtype]
        check(o, (w, (UNIT[g.dtype] + 2.0 ** -23 * (g.dtype is not F32)) * w.abs() * (1 + 2.0 ** -20) + tiny))
    if not stays:
        assert all(torch.equal(a, b) for a, b in zip(grads, given))


@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("stays", [False, True])
@pytest.mark.parametrize("most", [1e-3, 1.0, 1e9, math.inf, 0.0])
def test_clipping(most, stays, flat):
    check_clip(gradients(MANY, flat=flat), most, stays)
    check_clip(gradients([((100, 100), F32)]), most, stays)


def test_clipping_of_more_tensors_than_a_launch_takes():
    for n in (119, 120, 121, 1000):
        check_clip(gradients([((i % 7 * 40,), (F32, F16, BF16)[i % 3]) for i in range(n)]), 0.5, n % 2 == 0)
    check_clip(gradients([((5_000_000,), BF16), ((3_000_001,), F32)] * 2), 0.5, True)


def test_clipping_by_the_ends_of_the_numbers():
    L = lgp()
    check_clip([torch.full((1000,), 1e30, device="cuda"), torch.full((10,), -3e37, device="cuda")], 1.0, True)        # squares beyond fp32
    check_clip([torch.full((1000,), 1e-38, device="cuda")], 1e-39, True)
    check_clip([torch.full((10,), 60000.0, dtype=F16, device="cuda")], 60000.0, True)
    check_clip([torch.zeros(70, device="cuda")], 1.0, True)
    for bad in (math.inf, -math.inf, math.nan):
        g = [draw((3000,), F32, 1), draw((500,), BF16, 2)]
        g[1][77] = bad
        kept = [t.clone() for t in g]
        out = [torch.empty_like(t) for t in g]
        for o in (None, out):
            norm = L.clip_gradients(g, 0.1, out=o)
            assert not math.isfinite(float(norm))
            assert all(same(a, b) for a, b in zip(g, kept))
        assert all(same(a, b) for a, b in zip(out, kept))
    g = [torch.full((4,), 3e38, device="cuda")]                     # finite numbers whose norm is no float: left alone
    assert float(L.clip_gradients(g, 1.0)) == math.inf and (g[0] == 3e38).all()


def test_clipping_leaves_a_mark_for_autograd():
    L = lgp()
    w = torch.ones(5, device="cuda", requires_grad=True)
    g = torch.full((5,), 3.0, device="cuda")
    y = (w * g).sum()
    L.clip_gradients([g], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()


# ---- together

def test_a_training_step_of_the_second_half_of_a_layer():
    """The residual's addition and norm, the gated pair, the last projection (torch's), the next addition and norm; all gradients, and their clipping.  Along the way from the inputs
    to a gradient stand at most 14 roundings to fp16, each off by 2^-11 of what it rounds; the norms, the products and the activation's slope (1.13) hand an error on with no
    more than its share of what they hand on, but for cancellation, for which a factor of 3 is allowed."""
    L = lgp()
    T, W, H = 3000, 128, 200
    pos = slots(T, 1)
    live = pos >= 0
    leaf = dict(x=draw((T, W), F16, 2), res=draw((T, W), F32, 3, 2.0), n1=1 + draw((W,), F32, 4, 0.2), n2=1 + draw((W,), F32, 5, 0.2), wg=draw((H, W), F16, 6, W ** -0.5),
                wu=draw((H, W), F16, 7, W ** -0.5), wd=draw((W, H), F16, 8, H ** -0.5))
    leaf["x"][~live] = 0
    a, b = draw((T, W), F16, 9), draw((T, W), F32, 10)

    def step(v, norm, pair):
        y, total = norm(v["x"], v["res"], v["n1"])
        y, total = norm(pair(y, v["wg"], v["wu"]) @ v["wd"].t(), total, v["n2"])
        return y, total

    own = {n: t.clone().requires_grad_() for n, t in leaf.items()}
    y, total = step(own, lambda x, r, w: L.add_norm(x, r, w, pos=pos), lambda y, g, u: L.gated_linear(y, g, u, pos=pos))
    torch.autograd.backward([y, total], [a, b])

    def norm64(x, r, w):
        t = torch.where(live[:, None], x + r, 0.0)
        return torch.where(live[:, None], t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6) * w, 0.0), t

    exact = {n: t.double().requires_grad_() for n, t in leaf.items()}
    y64, total64 = step(exact, norm64, lambda y, g, u: torch.nn.functional.silu(y @ g.t()) * (y @ u.t()))
    torch.autograd.backward([y64, total64], [a.double(), b.double()])
    off = lambda g, w: float((g.detach().double() - w.detach()).norm() / w.detach().norm())  # noqa: E731
    assert off(y, y64) <= 5 * 3 * 2.0 ** -11 and off(total, total64) <= 4 * 3 * 2.0 ** -11
    for n in leaf:
        assert off(own[n].grad, exact[n].grad) <= 14 * 3 * 2.0 ** -11, n
    grads = [own[n].grad for n in leaf]
    before = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    assert abs(float(L.clip_gradients(grads, before / 3)) - before) <= 1e-6 * before
    after = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    assert abs(after - before / 3) <= 2.0 ** -11 * before / 3


# ---- streams, graphs, repeated runs

def pieces():
    x, res, w = draw((700, 256), BF16, 1), draw((700, 256), F32, 2), 1 + draw((256,), F32, 3, 0.1)
    wg, wu = draw((130, 248), BF16, 5, 0.06), draw((130, 248), BF16, 6, 0.06)
    wide = draw((90, 256), BF16, 7)
    pos = slots(700, 4)
    grads = gradients(MANY)
    out = [torch.empty_like(g) for g in grads]
    L = lgp()

    def run(stream=None):
        y, total = L.add_norm(x, res, w, pos=pos, stream=stream)
        back = L.add_norm_backward(y, total, total, w, pos=pos, stream=stream)
        rows, _ = L.add_norm_rows8(x, res, w, pos=pos, stream=stream)
        packed = L.pack_rows(x, pos=pos, stream=stream)
        h = L.gated_linear(y[:, :248], wg, wu, pos=pos, stream=stream)
        more = L.gated_linear_backward(h, y[:, :248], wg, wu, pos=pos, stream=stream)
        return [h, *more, y, total, *back, rows.values, rows.scales, packed.values, packed.scales, L.clip_gradients(grads, 0.3, out=out, stream=stream),
                *[o.clone() if stream is None else o for o in out]]
    return run, (x, res, *grads)


def test_runs_are_the_same_bit_by_bit():
    run, _ = pieces()
    first = run()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(), first))


def test_another_stream():
    run, _ = pieces()
    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_captured_and_replayed():
    run, inputs = pieces()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for seed in range(4):
        for t in inputs:
            t.copy_(draw(t.shape, t.dtype, 100 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [h.clone() for h in held]
        want = run()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


# ---- refusals

def test_refusals():
    L = lgp()
    x, w = torch.zeros(4, 32, dtype=BF16, device="cuda"), torch.ones(32, device="cuda")
    r8 = L.pack_rows(x)
    bad = [lambda: L.add_norm(x.cpu(), x, w), lambda: L.add_norm(x, x.half(), w), lambda: L.add_norm(x, x[:3], w), lambda: L.add_norm(x.float(), x, w),
           lambda: L.add_norm(x, x, w[:31]), lambda: L.add_norm(x, x, w.half()), lambda: L.add_norm(x, x, w, pos=torch.zeros(3, dtype=torch.int32, device="cuda")),
           lambda: L.add_norm(x, x, w, pos=torch.zeros(4, device="cuda")), lambda: L.add_norm(x.int(), None, w), lambda: L.add_norm(x[0], None, w),
           lambda: L.add_norm(x.t(), None, w[:4]), lambda: L.add_norm(x, x, w, eps=-1.0), lambda: L.add_norm(x, x, w, eps=1e300), lambda: L.add_norm(x, x, w.cpu()),
           lambda: L.add_norm(torch.zeros(1, 16385, device="cuda"), None, torch.ones(16385, device="cuda")),
           lambda: L.add_norm_backward(x, None, x.half(), w), lambda: L.add_norm_backward(x, x.float(), x, w), lambda: L.add_norm_backward(x[:2], None, x, w),
           lambda: L.add_norm_rows8(x, x.half(), w), lambda: L.pack_rows(x.int()), lambda: L.pack_rows(x.t()), lambda: L.pack_rows(torch.zeros(1, 16385, device="cuda")),
           lambda: L.Rows8(x, w, 32), lambda: L.Rows8(torch.zeros(4, 32, dtype=torch.int8, device="cuda"), w, 32),
           lambda: L.Rows8(torch.zeros(4, 20, dtype=torch.int8, device="cuda"), w[:4], 20),
           lambda: L.linear_rows8(r8, L.pack_rows(x[:, :24])), lambda: L.linear_rows8(r8, r8, bias=w[:3]), lambda: L.linear_rows8(r8, r8, bias=w[:4].half()),
           lambda: L.linear_rows8(r8, r8, dtype=torch.int8), lambda: L.linear_rows8(r8, L.pack_rows(x[:0])),
           lambda: L.linear_rows8(r8, L.pack_rows(x, pos=torch.zeros(4, dtype=torch.int32, device="cuda"))),
           lambda: L.gated_linear(x, x, x[:3]), lambda: L.gated_linear(x, x.half(), x), lambda: L.gated_linear(x, x[:, :24], x[:, :24]), lambda: L.gated_linear(x.float(), x, x),
           lambda: L.gated_linear(x, x, x, act="relu"), lambda: L.gated_linear(x[:, :20], x[:, :20].contiguous(), x[:, :20].contiguous()), lambda: L.gated_linear(x, x, x.cpu()),
           lambda: L.gated_linear(x[:, 4:12], x[:, :8].contiguous(), x[:, :8].contiguous()), lambda: L.gated_linear(x.t(), x, x), lambda: L.gated_linear(x, x[:0], x[:0]),
           lambda: L.gated_linear_backward(x, x[:2], x, x), lambda: L.gated_linear_backward(x[:, :2].float(), x, x[:2], x[:2]),
           lambda: L.clip_gradients([], 1.0), lambda: L.clip_gradients([x.t()], 1.0), lambda: L.clip_gradients([x.int()], 1.0), lambda: L.clip_gradients([x.cpu()], 1.0),
           lambda: L.clip_gradients([x], -1.0), lambda: L.clip_gradients([x], math.nan), lambda: L.clip_gradients([x], "one"), lambda: L.clip_gradients([x, x], 1.0),
           lambda: L.clip_gradients([x[:3], x[2:]], 1.0), lambda: L.clip_gradients([x[:2]], 1.0, out=[x[1:3]]), lambda: L.clip_gradients([x], 1.0, out=[x.half()]),
           lambda: L.clip_gradients([x, w], 1.0, out=[x]), lambda: L.clip_gradients([x, x.clone()], 1.0, out=[w.new_zeros(4, 32, dtype=BF16)] * 2),
           lambda: L.clip_gradients([x[:2], x[2:]], 1.0, out=[x[2:], x[:2]]), lambda: L.clip_gradients([x.cpu(), x], 1.0)]
    for i, call in enumerate(bad):
        with pytest.raises(L.LegionPrepError):
            call()
            pytest.fail(f"call {i} was taken")
    assert float(L.gradient_norm([x, x])) == 0.0                # only read: may be the same
    torch.cuda.synchronize()
