"""Operators of a model layer at the ends of their ranges, against their definitions in 64 bits (tests/layer_common.py)."""
import math
from types import SimpleNamespace

import pytest
import torch

import layer_common as ref
from test_gpu_9_layer import BF16, F16, F32, draw, lgp, make_docs, run_attention

pytestmark = pytest.mark.gpu


def alone(q, k, v, info, keep, **kw):
    """The definition over the keys that `keep` marks: the others have no weight at all, so the documents are as if they did not hold them."""
    at = torch.cat([torch.zeros(1, dtype=torch.long), keep.cpu().long().cumsum(0)])
    spans = [(qo, qn, int(at[ko]), int(at[ko + kn] - at[ko])) for qo, qn, ko, kn in info["spans"]]
    return ref.attention(q, k[keep], v[keep], dict(spans=spans, q_pos=info["q_pos"], k_pos=info["k_pos"][keep]), **kw)


# lengths that choose four waves of rows, four waves of keys, and one wave by itself; three tiles of keys and more each
SHAPES = [([300], [333]), ([20, 9], [200, 150]), ([40] * 5, [50] * 5)]


@pytest.mark.parametrize("q_owned,k_owned", SHAPES)
@pytest.mark.parametrize("dtype,dim", [(BF16, 32), (F16, 64), (BF16, 128)])
@pytest.mark.parametrize("nats", [60, 100, 300])
def test_scores_that_spread_widely(nats, dtype, dim, q_owned, k_owned):
    """Most keys of a row weigh nothing, and rows find their largest score in different tiles.  Probabilities below 2^-126 are zeros."""
    L = lgp()
    docs, info = make_docs(q_owned, k_owned)
    Tq, Tk = sum(q_owned), sum(k_owned)
    for heads, bias in ((2, False), (4, True)):
        q, k, v, g = (draw((t, h, dim), dtype, 1 + i, nats ** 0.5 if i < 2 else 1.0) for i, (t, h) in enumerate(((Tq, heads), (Tk, 2), (Tk, 2), (Tq, heads))))
        slopes = torch.linspace(0.05, 0.6, heads, device="cuda") if bias else None
        out, lse, rest = L.attend(q, k, v, docs, slopes=slopes, rest=True)
        got = L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, slopes=slopes)
        want = ref.attention(q, k, v, info, g, slopes)
        for x, name in zip((out, lse, *got[:3]), ("out", "lse", "dq", "dk", "dv")):
            value, bound = want[name]
            ref.check(x, (value, bound + 2.0 ** -110), name)


@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_rows,keys,late", [(70, 128, 100), (20, 400, 100), (20, 60, 50)])
def test_keys_that_weigh_nothing_in_every_other_four(q_rows, keys, late, dtype, half):
    """Four of eight keys lie 150 below the others, or have a score of -inf; one of a later tile is above all, so that some rows take a new base and
    all of them keep what they have."""
    L = lgp()
    at = torch.arange(keys, device="cuda")
    near = (at % 8 // 4 == half) & (at < late // 2)
    for low in (-150.0, -math.inf):
        score = torch.where(near, 5.40625, low)
        if half == 0:
            score[0] = 0.0                                     # the first base: the others are not far enough above for another
        score[late] = 5.8125 if half == 0 else 12.0
        q, k = torch.zeros((q_rows, 2, 64), device="cuda", dtype=dtype), torch.zeros((keys, 2, 64), device="cuda", dtype=dtype)
        q[:, :, 0] = 8.0
        q[1::2, :, 0] = 4.0                                    # in these rows the late key is not far above
        k[:, :, 0] = score[:, None].to(dtype)
        v = draw((keys, 2, 64), dtype, 3)
        docs, info = make_docs([q_rows], [keys])
        out, lse, _ = L.attend(q, k, v, docs, scale=0.125)
        want = alone(q, k, v, info, score > -math.inf, scale=0.125)
        ref.check(out, want["out"], f"out, {low}")
        ref.check(lse, want["lse"], f"lse, {low}")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim", [(1, 1, 1, 64), (5, 3, 1, 32), (1001, 5, 2, 128), (257, 1, 3, 40)])
def test_head_norms_without_eps(tokens, heads, kv_heads, dim, dtype):
    """Neither rows without a token nor places beyond the heads or the tokens are divided by a norm of zero."""
    L = lgp()
    q, k = draw((tokens, heads, dim), dtype, 1), draw((tokens, kv_heads, dim), dtype, 2)
    gq, gk = draw(q.shape, dtype, 3), draw(k.shape, dtype, 4)
    w = draw((dim,), F32, 5)
    pos, table = torch.arange(tokens, device="cuda", dtype=torch.int32), L.rotation_table(2000, 32)
    pos[1::3] = -1
    live = pos >= 0
    out = L.norm_rotate(q, k, w, w, pos, table, eps=0.0)
    back = L.norm_rotate_backward(gq, gk, q, k, w, w, pos, table, eps=0.0)
    for i, (x, g) in enumerate(((q, gq), (k, gk))):
        want = ref.head_norm(x[live], w, pos[live], table, 0.0, g[live])
        ref.check(out[i][live], want["out"], "out")
        ref.check(back[i][live], want["dx"], "dx")
        ref.check(back[2 + i], want["dw"], "dw")
        assert (out[i][~live] == 0).all() and (back[i][~live] == 0).all()


@pytest.mark.parametrize("x_dtype", [BF16, F32])
def test_weight_gradient_of_the_largest_activations(x_dtype):
    L = lgp()
    x = draw((70, 96), F32, 1)
    x[3, 32:64] *= 2.0 ** 126
    x[5, 0], x[6, 95] = torch.finfo(x_dtype).max, -torch.finfo(x_dtype).max
    dy = draw((70, 40), F32, 2, 2.0 ** -20).bfloat16()
    p = L.pack_activations(x.to(x_dtype))
    dw, _ = L.packed_weight_grad(p, dy)
    X, Y = L.unpack_activations(p).double(), dy.double()
    assert torch.isfinite(X).all()
    ref.check(dw, (Y.T @ X, 2.0 ** -24 * 72 * Y.abs().T @ X.abs()), "dw")


@pytest.mark.parametrize("q_owned,k_owned", SHAPES)
@pytest.mark.parametrize("far", [1e4, 1e6, 2.0 ** 24])
def test_keys_far_below_cost_the_others_no_digits(far, q_owned, k_owned):
    """A first key, or all keys of the first tiles, far below the rest, by their distance or by their product: in 64 bits they weigh nothing, and the
    others are as exact as without them."""
    L = lgp()
    Tq, Tk = sum(q_owned), sum(k_owned)
    q, k, v = draw((Tq, 4, 64), BF16, 1), draw((Tk, 2, 64), BF16, 2), draw((Tk, 2, 64), BF16, 3)
    for below in (1, min(k_owned) - 12):
        docs, info = make_docs(q_owned, k_owned)
        keep = torch.ones(Tk, dtype=torch.bool, device="cuda")
        for s in info["spans"]:
            keep[s[2]:s[2] + below] = False
        info["k_pos"][~keep] = int(far)                    # what docs holds too
        slopes = torch.linspace(1.0, 1.3, 4, device="cuda")
        out, lse, _ = L.attend(q, k, v, docs, slopes=slopes)
        want = alone(q, k, v, info, keep, slopes=slopes)
        ref.check(out, want["out"], "out, by distance")
        ref.check(lse, want["lse"], "lse, by distance")
        info["k_pos"].clamp_(max=7)
        k2, q2 = k.clone(), q.clone()
        q2[..., 0], k2[..., 0] = 1.0, 0.0
        k2[~keep] = 0
        k2[~keep, :, 0] = -8 * far
        out, lse, _ = L.attend(q2, k2, v, docs)
        want = alone(q2, k2, v, info, keep)
        ref.check(out, want["out"], "out, by product")
        ref.check(lse, want["lse"], "lse, by product")


def off(got, want):
    """Relative error in the 2-norm, and what rounding the exact result costs of it."""
    return float((got.double() - want).norm() / want.norm()), float((want.to(got.dtype).double() - want).norm() / want.norm())


@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("dim,rows", [(64, 300), (128, 40), (32, 33)])
def test_small_gradients_in_fp16(dim, rows, size):
    """dU = P (dP - delta) is far smaller than d_out over thousands of keys, and is rounded for the products that make dq and dk.  Beside the rounding
    of the result there are those of dU, of the probabilities in out (through delta) and of delta's sum, each at most a unit of the terms of the sum
    and at random: together less than four units."""
    L = lgp()
    keys = 6000
    docs, info = make_docs([rows], [keys])
    v, g = draw((keys, 2, dim), F16, 3), draw((rows, 2, dim), F32, 4, size).half()
    scale = 30 * dim ** -0.5
    for q_size, k_size in ((1 / 30, 1.0), (1.0, 1 / 30)):     # so that dq, and then dk, is not among the smallest numbers itself
        q, k = draw((rows, 2, dim), F16, 1, q_size), draw((keys, 2, dim), F16, 2, k_size)
        out, lse, rest = L.attend(q, k, v, docs, scale=scale, rest=True)
        got = L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, scale=scale)
        want = ref.attention(q, k, v, info, g, scale=scale)
        for x, name in zip(got, ("dq", "dk", "dv")):
            err, own = off(x, want[name][0])
            assert err <= own + 4 * ref.UNIT[F16], f"{name}: {err:.3g}, rounding alone {own:.3g}"


@pytest.mark.parametrize("dim,rows", [(64, 300), (128, 40), (32, 33)])
def test_large_gradients_in_fp16(dim, rows):
    """dU beyond the largest number of fp16, where dq, dk and dv are not, in some rows and in some tiles of the keys only."""
    L = lgp()
    keys = 200
    docs, info = make_docs([rows], [keys])
    q, k, v = draw((rows, 2, dim), F16, 1, 0.01), draw((keys, 2, dim), F16, 2, 0.01), draw((keys, 2, dim), F16, 3, 0.5)
    v[100:] *= 400
    g = draw((rows, 2, dim), F32, 4, 8000.0)
    g[::3] *= 1e-4
    g = g.half()
    out, lse, rest = L.attend(q, k, v, docs, rest=True)
    got = L.attend_backward(g, q, k, v, out, lse, docs, rest=rest)
    want = ref.attention(q, k, v, info, g)
    P = torch.softmax(q[:, 0].double() @ k[:, 0].double().T * dim ** -0.5, 1)
    dP = g[:, 0].double() @ v[:, 0].double().T
    assert (P * (dP - (P * dP).sum(1, keepdim=True))).abs().max() > 2 * 65504
    for x, name in zip(got, ("dq", "dk", "dv")):
        err, own = off(x, want[name][0])
        assert err <= own + 4 * ref.UNIT[F16], f"{name}: {err:.3g}, rounding alone {own:.3g}"


def test_the_largest_gradients_in_fp16_over_long_distances():
    """The sums for the slopes' gradient hold dU times distances of up to 2^24."""
    L = lgp()
    docs, info = make_docs([64], [128])
    info["k_pos"].copy_(torch.arange(128, device="cuda") * (1 << 17))
    q, k, v = draw((64, 2, 64), F16, 1, 0.1), draw((128, 2, 64), F16, 2, 0.1), draw((128, 2, 64), F16, 3, 60.0)
    g = draw((64, 2, 64), F32, 4, 12000.0).half()
    slopes = torch.full((2,), 1e-7, device="cuda")
    out, lse, rest = L.attend(q, k, v, docs, slopes=slopes, rest=True)
    ds = L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, slopes=slopes)[3]
    ref.check(ds, ref.attention(q, k, v, info, g, slopes)["d_slopes"], "d_slopes")


def milliseconds(f):
    f()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    f()
    b.record()
    b.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [(F16, 32, 4, 4), (BF16, 64, 4, 2), (BF16, 128, 3, 3)])
@pytest.mark.parametrize("large", [{700: (2000, 2000)}, {0: (1, 60_000), 1999: (300, 900)}, {d: (30, 40 + d % 50) for d in range(0, 1990, 37)},
                                   {5: (1, 513), 6: (2, 256), 7: (2, 257), 1500: (1900, 0), 1501: (0, 5000)}])
def test_large_documents_among_many_small_ones(large, dtype, dim, heads, kv_heads):
    """One query and few keys on average.  What has many of both is not one wave's work: a quarter of a second is ten times what the slowest of these
    cases takes, and a hundredth of four million pairs one after the other."""
    n = 2000
    rng = torch.Generator().manual_seed(1)
    small = torch.randint(0, 9, (n,), generator=rng).tolist()
    rest = n - sum(q for q, _ in large.values())               # queries that are left for the others
    q_owned, k_owned = [0] * n, list(small)
    for d, (q, k) in large.items():
        q_owned[d], k_owned[d] = q, k
    for d in range(n):
        if d not in large and rest > 0:
            q_owned[d], rest = 1, rest - 1
    q_tokens = [max(0, q - 3) if q > 50 else q for q in q_owned]
    docs, info = make_docs(q_owned, k_owned, q_tokens, [max(0, k - 5) if k > 50 else k for k in k_owned])
    run_attention(docs, info, heads, kv_heads, dim, dtype, 20.0, True)
    out, lse, dq, dk, dv, _ = run_attention(docs, info, heads, kv_heads, dim, dtype)
    L = lgp()
    q, k, g = (torch.zeros((t, h, dim), dtype=dtype, device="cuda") for t, h in ((sum(q_owned), heads), (sum(k_owned), kv_heads), (sum(q_owned), heads)))
    assert milliseconds(lambda: L.attend_backward(g, q, k, k, *L.attend(q, k, k, docs)[:2], docs)) < 250


def test_large_documents_in_graphs_and_twice():
    L = lgp()
    owned = [1] * 500
    owned[13], owned[400] = 90, 70
    for d in range(20, 180):
        owned[d] = 0
    docs, _ = make_docs(owned, [k + 9 for k in owned])
    Tq, Tk = sum(owned), sum(owned) + 9 * 500
    q, k, v, g = draw((Tq, 4, 64), BF16, 1), draw((Tk, 2, 64), BF16, 2), draw((Tk, 2, 64), BF16, 3), draw((Tq, 4, 64), BF16, 4)
    slopes = torch.full((4,), 0.1, device="cuda")

    def step():
        out, lse, rest = L.attend(q, k, v, docs, slopes=slopes, cap=30.0, rest=True)
        return [out, lse, rest, *L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, slopes=slopes, cap=30.0)]

    want = step()
    assert all(torch.equal(a, b) for a, b in zip(step(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for r in range(3):
        q.copy_(draw((Tq, 4, 64), BF16, 10 + r))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step())), f"replay {r}"


def test_many_large_documents_in_a_row():
    """More than a wave lists and goes through at once, at the ends of a long list of documents."""
    n = 40_000
    q_owned, k_owned = [0] * n, [2] * n
    for d in [*range(100), 511, 512, 513, 20_000, *range(n - 90, n)]:
        q_owned[d], k_owned[d] = 23, 24
    q_owned[30_000], q_owned[30_001] = 1, 1
    docs, info = make_docs(q_owned, k_owned)
    run_attention(docs, info, 2, 1, 32, F16, 20.0, True)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("cap,q_size,k_size,scale", [(1e6, 100.0, 1000.0, 1.0), (2e5, 30.0, 300.0, 1.0), (1e-6, 1.0, 1.0, 0.125), (1e-30, 1.0, 1.0, 0.125),
                                                     (1e-44, 1.0, 1.0, 0.125), (1e30, 1.0, 1.0, 0.125), (30.0, 1.0, 1.0, 0.0), (30.0, 1.0, 1.0, 1e-12)])
@pytest.mark.parametrize("q_owned,k_owned", [([70], [130]), ([1] * 20, [9] * 20)])
def test_caps_of_every_size(q_owned, k_owned, cap, q_size, k_size, scale, dtype):
    """The cap's tanh is a polynomial in the product where scores are near, with powers of scale / cap as coefficients.  Rows of zeros among the queries."""
    L = lgp()
    Tq, Tk = sum(q_owned), sum(k_owned)
    docs, info = make_docs(q_owned, k_owned)
    q, k, v, g = draw((Tq, 2, 32), dtype, 1, q_size), draw((Tk, 2, 32), dtype, 2, k_size), draw((Tk, 2, 32), dtype, 3), draw((Tq, 2, 32), dtype, 4)
    q[::4] = 0
    out, lse, rest = L.attend(q, k, v, docs, cap=cap, scale=scale, rest=True)
    got = L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, cap=cap, scale=scale)
    want = ref.attention(q, k, v, info, g, cap=cap, scale=scale)
    ref.check(out, want["out"], "out")
    ref.check(lse, want["lse"], "lse")
    for x, name in zip(got, ("dq", "dk", "dv")):
        value, bound = want[name]
        ref.check(x, (value, bound + 2.0 ** -110), name)


@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (16, 1), (3, 1), (2, 2)])
def test_heads_before_rows_in_long_lists(heads, kv_heads):
    """As lists that are kept by head have them: a head begins as far behind the one before as a long list is."""
    L = lgp()

    def by_head(t, apart):
        store = torch.empty((t.shape[1] - 1) * apart + t.shape[0] * t.shape[2], dtype=t.dtype, device="cuda")
        x = store.as_strided(t.shape, (t.shape[2], apart, 1))
        return x.copy_(t)

    for owned in ([290, 10], [1] * 300):
        docs, info = make_docs(owned, owned)
        q, k, v, g = (draw((300, h, 64), BF16, i) for i, h in enumerate((heads, kv_heads, kv_heads, heads)))
        far = (by_head(q, (1 << 25) + 64), by_head(k, (1 << 28) + 8), by_head(v, 1 << 24))
        near = L.attend(q, k, v, docs)[:2]
        assert all(torch.equal(a, b) for a, b in zip(L.attend(*far, docs), near))
        assert all(torch.equal(a, b) for a, b in zip(L.attend_backward(g, *far, *near, docs)[:3], L.attend_backward(g, q, k, v, *near, docs)[:3]))


def test_strides_of_a_single_row_or_head_say_nothing():
    L = lgp()
    docs, _ = make_docs([1], [1])
    x = draw((1, 3, 64), F16, 1)
    want = L.attend(x, x[:, :1], x[:, :1], docs)[:2]
    store = torch.empty(1 << 12, dtype=F16, device="cuda")
    for row in (77, 1 << 30):
        q, k = store.as_strided((1, 3, 64), (row, 64, 1)).copy_(x), store.as_strided((1, 1, 64), (row, 13, 1), 1024).copy_(x[:, :1])
        assert all(torch.equal(a, b) for a, b in zip(L.attend(q, k, k, docs), want))
        w = torch.ones(64, device="cuda")
        assert all(torch.equal(a, b) for a, b in zip(L.norm_rotate(q, k, w, w), L.norm_rotate(x, x[:, :1], w, w)))


def test_numbers_and_streams_that_do_not_fit_are_refused():
    L = lgp()
    docs, _ = make_docs([4], [4])
    q, w = draw((4, 2, 64), F16, 1), torch.ones(64, device="cuda")
    x = torch.ones((4, 8), device="cuda")
    elsewhere = SimpleNamespace(device_index=1, cuda_stream=0)
    for f in (lambda: L.attend(q, q, q, docs, cap=1e39), lambda: L.attend(q, q, q, docs, scale=-1e300), lambda: L.attend(q, q, q, docs, scale="1"),
              lambda: L.norm_rotate(q, q, w, w, eps=1e39), lambda: L.attend(q, q, q, docs, stream=elsewhere), lambda: L.norm_rotate(q, q, w, w, stream=elsewhere),
              lambda: L.pack_activations(x, stream=elsewhere)):
        with pytest.raises(L.LegionPrepError):
            f()


@pytest.mark.parametrize("side", [False, True])
def test_gradients_pass_through_the_operators(side):
    """What autograd makes of attend and norm_rotate is what their backward calls return, on the current stream and on another."""
    L = lgp()
    docs, info = make_docs([40, 1, 200], [40, 1, 200], [33, 1, 200], [33, 1, 200])
    qkv = draw((241, 8, 64), BF16, 1).requires_grad_()
    wq, wk, slopes = (draw((n,), F32, 2 + i).abs().requires_grad_() for i, n in enumerate((64, 64, 4)))
    pos, table = torch.arange(241, device="cuda", dtype=torch.int32), L.rotation_table(300, 32)
    g = draw((241, 4, 64), BF16, 5)
    stream = torch.cuda.Stream() if side else None
    if side:
        stream.wait_stream(torch.cuda.current_stream())
    q, k = L.norm_rotate(qkv[:, :4], qkv[:, 4:6], wq, wk, pos, table, stream=stream)
    out, lse, rest = L.attend(q, k, qkv[:, 6:], docs, slopes=slopes, cap=20.0, stream=stream)
    assert out.requires_grad and not lse.requires_grad and rest is None
    if side:
        torch.cuda.current_stream().wait_stream(stream)
    out.backward(g)
    torch.cuda.synchronize()
    with torch.no_grad():
        args = (qkv[:, :4], qkv[:, 4:6], wq, wk, pos, table)
        q2, k2 = L.norm_rotate(*args)
        out2, lse2, rest2 = L.attend(q2, k2, qkv[:, 6:], docs, slopes=slopes, cap=20.0, rest=True)
        assert not out2.requires_grad and torch.equal(out2, out) and torch.equal(lse2, lse)
        dq, dk, dv, ds = L.attend_backward(g, q2, k2, qkv[:, 6:], out2, lse2, docs, rest=rest2, slopes=slopes, cap=20.0)
        dq, dk, dwq, dwk = L.norm_rotate_backward(dq, dk, *args)
    assert torch.equal(qkv.grad, torch.cat([dq, dk, dv], 1)) and torch.equal(slopes.grad, ds) and torch.equal(wq.grad, dwq) and torch.equal(wk.grad, dwk)
    assert not L.unpack_activations(L.pack_activations(qkv.flatten(1))).requires_grad


@pytest.fixture
def room():
    """Most of the GPU's memory."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_head_norms_of_more_rows_than_a_launch_has_threads(room):
    """134 million rows of 32 lanes each; all but two of them are one row in memory."""
    L = lgp()
    T, at = (1 << 27) + 5, (1 << 26) + 3
    rows = draw((2, 1, 256), F16, 1)
    q, none = rows[:1].expand(T, 1, 256), torch.empty((T, 0, 256), dtype=F16, device="cuda")
    w = draw((256,), F32, 2)
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    pos[at], pos[T - 1] = 7, -1
    table = L.rotation_table(8, 64)
    out = L.norm_rotate(q, none, w, w, pos, table)[0]
    want = L.norm_rotate(rows[:1].expand(3, 1, 256).contiguous(), none[:3], w, w, pos[[0, at, T - 1]], table)[0]
    assert torch.equal(out[[0, at, T - 1]], want)
    out[at], out[T - 1] = want[0], want[0]
    assert all((part == want[0]).all() for part in out.split(1 << 24))


def test_packing_of_more_rows_than_a_launch_has_threads(room):
    L = lgp()
    T = (1 << 31) - 1                                           # 147 GB of results
    x = draw((1, 64), F16, 1)
    p = L.pack_activations(x.expand(T, 64))
    want = L.pack_activations(x)
    for got, one in ((p.values, want.values), (p.exps, want.exps)):
        assert all((part == one).all() for part in got.split(1 << 26))


def test_documents_of_more_tiles_than_a_launch_has_threads(room):
    """2.2 million documents of two rows, 32 heads: a wave each for 75 million tiles."""
    L = lgp()
    n, H, D = 2_200_000, 32, 8
    offs = torch.arange(n + 1, dtype=torch.int32, device="cuda") * 2
    docs = L.Documents(offs, offs)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, d_out = (torch.randn((2 * n, H, D), generator=g, device="cuda", dtype=F16) for _ in range(4))
    out, lse, rest = L.attend(q, k, v, docs, rest=True)
    got = out, *L.attend_backward(d_out, q, k, v, out, lse, docs, rest=rest)[:3]
    for d in (0, n // 2, n - 50_000):
        rows = slice(2 * d, 2 * d + 100_000)
        a, b, c, e = (t[rows].view(-1, 2, H, D).float().transpose(1, 2) for t in (q, k, v, d_out))
        P = torch.softmax((a[:, :, :, None] * b[:, :, None]).sum(-1) * D ** -0.5, 3)                # [documents, H, 2, 2]
        o = (P[..., None] * c[:, :, None]).sum(3)
        dS = P * ((e[:, :, :, None] * c[:, :, None]).sum(-1) - (e * o).sum(-1, keepdim=True)) * D ** -0.5
        want = o, (dS[..., None] * b[:, :, None]).sum(3), (dS[..., None] * a[:, :, :, None]).sum(2), (P[..., None] * e[:, :, :, None]).sum(2)
        for x, y, name in zip(got, want, ("out", "dq", "dk", "dv")):
            # terms of up to 40, a few units each
            assert (x[rows].view(-1, 2, H, D).float().transpose(1, 2) - y).abs().max() < 40 * 4 * ref.UNIT[F16], f"{name}, document {d}"


@pytest.mark.parametrize("q_owned,k_owned", [*SHAPES, ([1] * 60, [9] * 60)])
@pytest.mark.parametrize("dtype,size", [(F16, 1.2e4), (BF16, 1e9), (BF16, 1e-9)])
@pytest.mark.parametrize("bias", [False, True])
def test_scores_of_every_magnitude(bias, dtype, size, q_owned, k_owned):
    """Beyond 2^24 a score's place is more than the distance that a weight is lost over: a row's result is the value of its largest score, where that is
    larger by more than the rounding of the sums."""
    L = lgp()
    docs, info = make_docs(q_owned, k_owned)
    Tq, Tk = sum(q_owned), sum(k_owned)
    q, k, v = draw((Tq, 2, 128), dtype, 1, size), draw((Tk, 2, 128), dtype, 2, size), draw((Tk, 2, 128), dtype, 3)
    slopes = torch.full((2,), 0.1, device="cuda") if bias else None
    out, lse, _ = L.attend(q, k, v, docs, slopes=slopes, scale=1.0)
    assert torch.isfinite(out).all()
    want = ref.attention(q, k, v, info, None, slopes, scale=1.0)
    if size < 1:
        ref.check(out, want["out"], "out")
        ref.check(lse, want["lse"], "lse")
        return
    for qo, qn, ko, kn in info["spans"]:
        z = torch.matmul(q[qo:qo + qn].double().transpose(0, 1), k[ko:ko + kn].double().permute(1, 2, 0).contiguous())          # [heads, queries, keys]
        top = z.topk(2, 2)
        clear = ((top.values[..., 0] - top.values[..., 1]) > 2.0 ** -20 * 128 * float(z.abs().max())).t()
        best = torch.stack([v[ko:ko + kn, h][top.indices[h, :, 0]] for h in range(2)], 1)
        assert clear.float().mean() > 0.9 and torch.equal(out[qo:qo + qn][clear], best[clear])
        assert ((lse[qo:qo + qn].double() / top.values[..., 0].t() - 1).abs()[clear] < 2.0 ** -17).all()


@pytest.mark.parametrize("q_owned,k_owned", [([0], [1500]), ([0, 0], [9000, 2000]), ([0] * 50, [700] * 50)])
def test_keys_without_any_queries(q_owned, k_owned):
    """As many keys as are split where queries are few, and none of them."""
    docs, info = make_docs(q_owned, k_owned)
    for heads, kv_heads in ((2, 2), (8, 2)):
        _, _, _, dk, dv, ds = run_attention(docs, info, heads, kv_heads, 64, F16, 0.0, True)
        assert (dk == 0).all() and (dv == 0).all() and (ds == 0).all()
