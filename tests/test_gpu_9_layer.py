"""Operators of a model layer over sampled neighbourhoods against their definitions in 64 bits (tests/layer_common.py), at the sizes, masks and layouts
where they can go wrong; their refusals; streams, captured graphs and runs that are repeated bit by bit."""
import math

import numpy as np
import pytest
import torch

import layer_common as ref

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def lgp():
    import paper_2305_16588_amd
    return paper_2305_16588_amd


def make_docs(q_owned, k_owned, q_tokens=None, k_tokens=None, seed=0, hops=8):
    """Documents of these row counts, on the GPU: (Documents, what the reference wants)."""
    def side(owned, tokens):
        offs = torch.tensor([0] + owned).cumsum(0).to(torch.int32)
        return offs, None if tokens is None else torch.tensor(tokens, dtype=torch.int32)

    g = torch.Generator().manual_seed(seed)
    (qo, qt), (ko, kt) = side(q_owned, q_tokens), side(k_owned, k_tokens)
    q_pos, k_pos = (torch.randint(0, hops, (int(o[-1]),), generator=g, dtype=torch.int32).cuda() for o in (qo, ko))
    spans = [(int(qo[d]), (q_tokens or q_owned)[d], int(ko[d]), (k_tokens or k_owned)[d]) for d in range(len(q_owned))]
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    docs = lgp().Documents(cu(qo), cu(ko), q_lens=cu(qt), k_lens=cu(kt), q_pos=q_pos, k_pos=k_pos)
    return docs, dict(spans=spans, q_pos=q_pos, k_pos=k_pos)


def draw(shape, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * size).to(dtype)


def hide(t, spans, which):
    """NaN in the rows that hold no token."""
    seen = torch.zeros(t.shape[0], dtype=torch.bool, device=t.device)
    for s in spans:
        at, n = (s[0], s[1]) if which == "q" else (s[2], s[3])
        seen[at:at + n] = True
    t[~seen] = math.nan


def run_attention(docs, info, heads, kv_heads, dim, dtype, cap=0.0, bias=False, seed=1, size=1.0, rest=True, hidden=True, scale=None):
    L = lgp()
    Tq, Tk = info["q_pos"].numel(), info["k_pos"].numel()
    q, k, v, g = (draw((t, h, dim), dtype, seed + i, size if i < 2 else 1.0) for i, (t, h) in enumerate(((Tq, heads), (Tk, kv_heads), (Tk, kv_heads), (Tq, heads))))
    if hidden:
        for t, which in ((q, "q"), (g, "q"), (k, "k"), (v, "k")):
            hide(t, info["spans"], which)
    slopes = torch.linspace(0.05, 0.6, heads, device="cuda") if bias else None
    out, lse, left = L.attend(q, k, v, docs, slopes=slopes, cap=cap, scale=scale, rest=rest)
    dq, dk, dv, ds = L.attend_backward(g, q, k, v, out, lse, docs, rest=left, slopes=slopes, cap=cap, scale=scale)
    want = ref.attention(q, k, v, info, g, slopes, cap, scale, exact_delta=rest)
    ref.check(out, want["out"], "out")
    ref.check(lse, want["lse"], "lse")
    ref.check(dq, want["dq"], "dq")
    ref.check(dk, want["dk"], "dk")
    ref.check(dv, want["dv"], "dv")
    if bias:
        ref.check(ds, want["d_slopes"], "d_slopes")
    return out, lse, dq, dk, dv, ds


EDGES = [0, 1, 2, 7, 16, 31, 32, 33, 40, 63, 64, 65, 0, 96, 127, 128, 129, 200, 257, 1]


@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (20.0, True)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 2, 2), (32, 3, 1), (128, 4, 2), (8, 1, 1), (40, 2, 1), (104, 2, 2), (56, 5, 5)])
def test_documents_of_every_length(dim, heads, kv_heads, dtype, cap, bias):
    rng = np.random.default_rng(dim)
    for own in (True, False):        # queries and keys of the same rows' counts, and of counts that have nothing to do with each other
        ks = EDGES if own else rng.permutation(EDGES).tolist()
        docs, info = make_docs(EDGES, ks)
        run_attention(docs, info, heads, kv_heads, dim, dtype, cap, bias)


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [(F16, 32, 8, 8), (BF16, 64, 8, 2), (F16, 24, 4, 1)])
def test_lists_of_a_frontier(dtype, dim, heads, kv_heads):
    """Single queries over up to 15 slots, as the sampler lists them; slots without a sample hold NaN, some vertices have none at all."""
    rng = np.random.default_rng(7)
    for n in (1, 63, 1000):
        tokens = rng.integers(0, 16, n).tolist()
        docs, info = make_docs([1] * n, [15] * n, None, tokens)
        run_attention(docs, info, heads, kv_heads, dim, dtype, 30.0, True)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_slots_on_both_sides(dtype):
    docs, info = make_docs([40, 7, 300, 1, 0, 130, 5], [40, 7, 300, 1, 0, 130, 5], [33, 0, 255, 1, 0, 128, 5], [33, 0, 255, 1, 0, 128, 5])
    out, lse, dq, dk, dv, _ = run_attention(docs, info, 4, 2, 64, dtype, 30.0, True)
    assert (out[33:47] == 0).all() and torch.isinf(lse[33:47]).all() and (dq[33:47] == 0).all() and (dk[33:47] == 0).all() and (dv[33:47] == 0).all()


@pytest.mark.parametrize("lens", [[1], [256], [511, 513], [5000], [20_000, 0, 1, 7777], [3000] * 5])
@pytest.mark.parametrize("dtype,heads,kv_heads,dim", [(BF16, 16, 2, 128), (F16, 4, 4, 64), (BF16, 40, 1, 40)])
def test_few_queries_over_long_lists(lens, dtype, heads, kv_heads, dim):
    docs, info = make_docs([1] * len(lens), lens)
    run_attention(docs, info, heads, kv_heads, dim, dtype, 0.0, True, size=1.5)
    docs, info = make_docs([3] * len(lens), lens)
    run_attention(docs, info, heads, kv_heads, dim, dtype, 25.0, False)


def test_one_long_document():
    docs, info = make_docs([3001], [2999])
    run_attention(docs, info, 2, 1, 64, BF16, 0.0, True)
    run_attention(docs, info, 2, 2, 128, F16, 50.0, False, rest=False)


def test_sharp_scores_and_scales():
    docs, info = make_docs([70, 200], [90, 150])
    for size in (6.0, 0.01):
        run_attention(docs, info, 2, 2, 64, BF16, size=size)
        run_attention(docs, info, 2, 2, 64, F16, 10.0, size=size)
    run_attention(docs, info, 2, 2, 64, F16, scale=-0.3)
    run_attention(docs, info, 2, 2, 64, BF16, scale=0.0)


def test_nothing_to_do():
    L = lgp()
    for q_owned, k_owned in (([], []), ([0, 0], [0, 0]), ([0], [70]), ([70], [0]), ([1], [0])):
        docs, info = make_docs(q_owned, k_owned)
        out, lse, dq, dk, dv, ds = run_attention(docs, info, 4, 2, 64, F16, 0.0, True)
        assert (out == 0).all() and torch.isinf(lse).all() and (dk == 0).all() and (dv == 0).all() and (ds == 0).all()
    packed = L.pack_activations(torch.empty((0, 40), dtype=F16, device="cuda"))
    assert L.unpack_activations(packed).shape == (0, 40)
    dw, db = L.packed_weight_grad(packed, torch.empty((0, 24), dtype=F16, device="cuda"))
    assert dw.shape == (24, 40) and (dw == 0).all() and (db == 0).all()
    q, k = torch.empty((0, 4, 64), dtype=F16, device="cuda"), torch.empty((0, 2, 64), dtype=F16, device="cuda")
    w = torch.ones(64, device="cuda")
    assert L.norm_rotate(q, k, w, w)[0].shape == (0, 4, 64)
    assert all((x == 0).all() for x in L.norm_rotate_backward(q, k, q, k, w, w)[2:])


def test_infinities_and_nan_stay_where_they_belong():
    """A value that is not finite reaches the rows of its document and no other."""
    L = lgp()
    docs, info = make_docs([40, 40, 40], [50, 50, 50])
    q, k, v = draw((120, 2, 64), BF16, 1), draw((150, 2, 64), BF16, 2), draw((150, 2, 64), BF16, 3)
    clean, clean_lse, _ = L.attend(q, k, v, docs)
    k[60, 0, 3], v[70, 1, 5], v[75, 1, 6] = math.nan, math.nan, math.inf
    out, lse, _ = L.attend(q, k, v, docs)
    assert torch.isnan(out[40:80, 0]).all() and torch.isnan(lse[40:80, 0]).all()
    assert torch.isnan(out[40:80, 1, 5]).all() and (out[40:80, 1, 6] == math.inf).all()
    rows = torch.cat([torch.arange(40), torch.arange(80, 120)])
    assert torch.equal(out[rows], clean[rows]) and torch.equal(lse[rows], clean_lse[rows]) and torch.equal(lse[40:80, 1], clean_lse[40:80, 1])
    # scores of -inf are masked places: a document in which all are leaves its queries without keys
    docs, info = make_docs([3, 3], [40, 40])
    q, k, v = torch.ones((6, 1, 32), dtype=F16, device="cuda"), draw((80, 1, 32), F16, 2), draw((80, 1, 32), F16, 3)
    k[:40] = -65504.0
    k[:40, :, 0] = -math.inf
    k[41:80, :, 0] = -math.inf
    out, lse, rest = L.attend(q, k, v, docs, rest=True)
    assert (out[:3] == 0).all() and (lse[:3] == -math.inf).all()
    assert torch.equal(out[3:], v[40].expand(3, 1, 32))
    # the lowest value of the type is a number like others
    k = torch.full((80, 1, 32), -65504.0, dtype=F16, device="cuda")
    out, lse, _ = L.attend(q, k, v, docs)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert torch.allclose(out[0, 0].float(), v[:40, 0].float().mean(0), atol=2e-3)


def test_strided_inputs():
    """Views into one product's result, heads before rows, and gaps between rows."""
    L = lgp()
    docs, info = make_docs([33, 100, 1], [33, 100, 1])
    x = draw((134, 4 + 2 * 2, 64), BF16, 5)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    want = L.attend(q.contiguous(), k.contiguous(), v.contiguous(), docs)[:2]
    for got in (L.attend(q, k, v, docs), L.attend(q.transpose(0, 1).contiguous().transpose(0, 1), k.transpose(0, 1).contiguous().transpose(0, 1), v, docs)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = draw((134, 4, 64), BF16, 6)
    a = L.attend_backward(g, q, k, v, *want, docs)
    b = L.attend_backward(g.transpose(0, 1).contiguous().transpose(0, 1), q.contiguous(), k.contiguous(), v.contiguous(), *want, docs)
    assert all(torch.equal(s, t) for s, t in zip(a[:3], b[:3]))


def test_keys_beyond_32_bits_of_offset():
    """Rows so far apart that their place in memory does not fit 32 bits, in elements."""
    L = lgp()
    stride = 8_000_000                                           # 300 rows of it: 2.4 * 10^9 elements
    store = torch.empty(300 * stride, dtype=F16, device="cuda")
    k, v = (store.as_strided((300, 2, 64), (stride, 64, 1), at) for at in (0, 4096))
    k.copy_(draw((300, 2, 64), F16, 1))
    v.copy_(draw((300, 2, 64), F16, 2))
    q = store.as_strided((300, 2, 64), (stride, 64, 1), 8192)
    q.copy_(draw((300, 2, 64), F16, 3))
    for owned in ([299, 1], [10] * 30):
        docs, info = make_docs(owned, owned)
        g = draw((300, 2, 64), F16, 4)
        far = L.attend(q, k, v, docs)[:2]
        near = L.attend(q.contiguous(), k.contiguous(), v.contiguous(), docs)[:2]
        assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
        a, b = L.attend_backward(g, q, k, v, *far, docs), L.attend_backward(g, q.contiguous(), k.contiguous(), v.contiguous(), *near, docs)
        assert all(torch.equal(s, t) for s, t in zip(a[:3], b[:3]))


def test_offsets_that_make_no_sense_touch_nothing_else():
    """Descending, negative and too large offsets and counts: whatever comes out, only the results are written."""
    L = lgp()
    q, k, v = draw((100, 2, 64), F16, 1), draw((100, 2, 64), F16, 2), draw((100, 2, 64), F16, 3)
    for offs in ([0, 70, 30, 100], [5, -4, 2000, 7], [0, 2 ** 31 - 1, -2 ** 31, 50]):
        o = torch.tensor(offs, dtype=torch.int32, device="cuda")
        n = torch.tensor([-3, 2 ** 31 - 1, 20], dtype=torch.int32, device="cuda")
        docs = L.Documents(o, o, q_lens=n, k_lens=n)
        out, lse, _ = L.attend(q, k, v, docs)
        L.attend_backward(q, q, k, v, out, lse, docs)
    torch.cuda.synchronize()


def test_attention_is_the_same_every_time_on_streams_and_in_graphs():
    L = lgp()
    docs, info = make_docs([200, 1, 64, 0, 500], [300, 9000, 64, 5, 0])
    q, k, v, g = draw((765, 4, 64), BF16, 1), draw((9369, 2, 64), BF16, 2), draw((9369, 2, 64), BF16, 3), draw((765, 4, 64), BF16, 4)
    slopes = torch.full((4,), 0.1, device="cuda")

    def step(stream=None):
        out, lse, rest = L.attend(q, k, v, docs, slopes=slopes, cap=30.0, rest=True, stream=stream)
        return [out, lse, rest, *L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, slopes=slopes, cap=30.0, stream=stream)]

    want = step()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for r in range(3):
        q.copy_(draw((765, 4, 64), BF16, 10 + r))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step())), f"replay {r}"


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim,rot", [(8, 0), (16, 16), (24, 16), (32, 32), (64, 32), (72, 64), (128, 128), (136, 16), (256, 256), (248, 240)])
@pytest.mark.parametrize("tokens,heads,kv_heads", [(1, 1, 1), (3, 5, 2), (1000, 4, 4), (257, 8, 1)])
def test_head_norms(tokens, heads, kv_heads, dim, rot, dtype):
    L = lgp()
    qkv = draw((tokens, heads + 2 * kv_heads, dim), dtype, dim + tokens)
    pos = torch.randint(0, 500, (tokens,), device="cuda", dtype=torch.int32)
    pos[::7] = 499
    if tokens > 1:
        pos[1::5] = -1
        pos[tokens - 1] = 2 ** 31 - 1                  # beyond the table
        qkv[pos < 0] = math.nan
    table = L.rotation_table(500, rot) if rot else None
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv_heads]
    wq, wk = draw((dim,), F32, 3), draw((dim,), F32, 4)
    gq, gk = draw(q.shape, dtype, 5), draw(k.shape, dtype, 6)
    gq[pos < 0], gk[pos < 0] = math.nan, math.nan
    got = L.norm_rotate(q, k, wq, wk, pos, table, eps=1e-5)
    back = L.norm_rotate_backward(gq, gk, q, k, wq, wk, pos, table, eps=1e-5)
    for i, (x, w, g) in enumerate(((q, wq, gq), (k, wk, gk))):
        want = ref.head_norm(x, w, pos, table, 1e-5, g)
        ref.check(got[i], want["out"], "out")
        ref.check(back[i], want["dx"], "dx")
        ref.check(back[2 + i], want["dw"], "dw")
    if not rot:
        none = L.norm_rotate(q, k, wq, wk, eps=1e-5)          # without positions every row is a token
        assert torch.equal(none[0][pos >= 0], got[0][pos >= 0])


def test_head_norms_of_many_rows_and_of_zeros():
    L = lgp()
    T = 40_003
    q, k = draw((T, 3, 64), BF16, 1, 3.0), draw((T, 3, 64), BF16, 2, 1e-3)
    q[5] = 0
    w = draw((64,), F32, 3)
    g = draw((T, 3, 64), BF16, 4)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) % 300
    table = L.rotation_table(300, 64)
    got, back = L.norm_rotate(q, k, w, w, pos, table), L.norm_rotate_backward(g, g, q, k, w, w, pos, table)
    for i, x in enumerate((q, k)):
        want = ref.head_norm(x, w, pos, table, 1e-6, g)
        ref.check(got[i], want["out"], "out")
        ref.check(back[i], want["dx"], "dx")
        ref.check(back[2 + i], want["dw"], "dw")
    assert (got[0][5] == 0).all()
    again = L.norm_rotate_backward(g, g, q, k, w, w, pos, table)
    assert all(torch.equal(a, b) for a, b in zip(again, back))


def test_rotation_table():
    L = lgp()
    t = L.rotation_table(1000, 32, base=500.0)
    i, p = 5, 777
    assert t.shape == (1000, 32) and abs(t[p, i].item() - math.cos(p * 500.0 ** (-2 * i / 32))) < 1e-7 and abs(t[p, 16 + i].item() - math.sin(p * 500.0 ** (-2 * i / 32))) < 1e-7


def awkward(tokens, width, dtype, seed):
    """Values of very different sizes, ties, subnormal numbers, the largest ones, zeros, and groups that are not finite."""
    x = draw((tokens, width), F32, seed) * torch.exp2(torch.randint(-12, 10, (tokens, 1), device="cuda").float())
    x[::5] = torch.randint(-260, 261, x[::5].shape, device="cuda").float() / 2            # ties of a step of one
    x = x.to(dtype)
    if tokens > 12:
        x[2] = torch.finfo(dtype).tiny / 8
        x[3] = torch.finfo(dtype).max * torch.where(torch.arange(width, device="cuda") % 2 == 0, 1.0, -0.999).to(dtype)
        x[4] = 0
        x[7, width // 2] = math.inf
        x[8, width - 1] = math.nan
        x[9, 0] = -math.inf
        x[11] = 127.9 / 64
    return x


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("tokens,width", [(1, 1), (13, 7), (40, 31), (17, 32), (33, 33), (20, 100), (64, 128), (5, 1000), (300, 8), (14, 257)])
def test_packing(tokens, width, dtype):
    L = lgp()
    x = awkward(tokens, width, dtype, width)
    values, exps, held = ref.pack(x)
    p = L.pack_activations(x)
    assert torch.equal(p.values.cpu(), values) and torch.equal(p.exps.cpu(), exps)
    back = L.unpack_activations(p)
    assert back.dtype == dtype and torch.equal(torch.isnan(back.cpu()), torch.isnan(held)) and torch.equal(back.double().cpu().nan_to_num(9e9), held.nan_to_num(9e9))
    # a view that is aligned to nothing but its elements, and rows without a token
    wide = torch.full((tokens, width + 3), math.nan, dtype=dtype, device="cuda")
    wide[:, 1:1 + width] = x
    pos = torch.arange(tokens, device="cuda", dtype=torch.int32)
    pos[::3] = -1
    p = L.pack_activations(wide[:, 1:1 + width], pos=pos)
    values, exps, held = ref.pack(x, pos)
    assert torch.equal(p.values.cpu(), values) and torch.equal(p.exps.cpu(), exps)


@pytest.mark.parametrize("x_dtype,dtype", [(F16, F16), (BF16, BF16), (F32, BF16), (F16, BF16)])
@pytest.mark.parametrize("tokens,width,out", [(1, 1, 1), (5, 8, 3), (63, 100, 256), (64, 128, 128), (65, 129, 127), (1000, 257, 72), (6000, 40, 200), (333, 512, 384)])
def test_weight_gradient(tokens, width, out, x_dtype, dtype):
    L = lgp()
    x = draw((tokens, width), F32, 1).mul_(torch.exp2(torch.randint(-6, 6, (1, width), device="cuda").float())).to(x_dtype)
    pos = torch.arange(tokens, device="cuda", dtype=torch.int32)
    if tokens > 4:
        pos[1::4] = -1
        x[pos < 0] = math.nan
    store = draw((tokens, out + 5), dtype, 2)
    dy = store[:, 2:2 + out]                                 # neither aligned nor end to end
    dy[pos < 0] = math.nan
    p = L.pack_activations(x, pos=pos)
    dw, db = L.packed_weight_grad(p, dy)
    X, Y = L.unpack_activations(p).double(), torch.where((pos >= 0)[:, None], dy.double(), 0.0)
    e = 2.0 ** -24 * (tokens + 2)                            # every sum of n numbers in fp32, whatever its order
    ref.check(dw, (Y.T @ X, e * Y.abs().T @ X.abs()), "dw")
    ref.check(db, (Y.sum(0), e * Y.abs().sum(0)), "db")
    again = L.packed_weight_grad(p, dy.contiguous(), bias=False)
    assert torch.equal(again[0], dw) and again[1] is None


def test_weight_gradient_of_long_sums():
    """Many parts of the tokens: split, added in their order, and the same every time."""
    L = lgp()
    T = 100_001
    x, dy = draw((T, 72), F16, 1), draw((T, 136), F16, 2)
    p = L.pack_activations(x)
    dw, db = L.packed_weight_grad(p, dy)
    X, Y = L.unpack_activations(p).double(), dy.double()
    e = 2.0 ** -24 * 1500           # no sum in a row is longer: of a part's tokens, 16 at a time, or of the parts
    ref.check(dw, (Y.T @ X, e * Y.abs().T @ X.abs()), "dw")
    ref.check(db, (Y.sum(0), e * Y.abs().sum(0)), "db")
    assert all(torch.equal(a, b) for a, b in zip(L.packed_weight_grad(p, dy), (dw, db)))


def test_a_group_that_is_not_finite_is_seen_in_the_gradient():
    L = lgp()
    x, dy = draw((70, 64), F16, 1), draw((70, 40), F16, 2)
    x[9, 40] = math.inf
    p = L.pack_activations(x)
    dw, db = L.packed_weight_grad(p, dy)
    assert torch.isnan(dw[:, 32:]).all() and torch.isfinite(dw[:, :32]).all() and torch.isfinite(db).all()


def test_norms_and_packing_in_graphs_and_on_streams():
    L = lgp()
    x, dy = draw((3000, 200), BF16, 1), draw((3000, 96), BF16, 2)
    q, k, w = draw((500, 4, 64), BF16, 3), draw((500, 2, 64), BF16, 4), draw((64,), F32, 5)
    pos, table = torch.arange(500, device="cuda", dtype=torch.int32), L.rotation_table(500, 32)

    def step(stream=None):
        p = L.pack_activations(x, stream=stream)
        return [p.values, p.exps, L.unpack_activations(p, stream=stream), *L.packed_weight_grad(p, dy, stream=stream),
                *L.norm_rotate(q, k, w, w, pos, table, stream=stream), *L.norm_rotate_backward(q, k, q, k, w, w, pos, table, stream=stream)]

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for r in range(3):
        x.copy_(draw((3000, 200), BF16, 10 + r))
        q.copy_(draw((500, 4, 64), BF16, 20 + r))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step())), f"replay {r}"


def test_refusals():
    L = lgp()
    docs, _ = make_docs([4, 4], [4, 4])
    q, k = draw((8, 4, 64), F16, 1), draw((8, 2, 64), F16, 2)
    w = torch.ones(64, device="cuda")
    o = torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [
        lambda: L.attend(q.float(), k.float(), k.float(), docs),                         # types
        lambda: L.attend(q, k.bfloat16(), k, docs),
        lambda: L.attend(q[:, :3], k, k, docs),                                          # 3 heads over 2
        lambda: L.attend(q[:, :, :60], k[:, :, :60], k[:, :, :60], docs),                # a dimension of 60
        lambda: L.attend(draw((8, 2, 136), F16, 1), draw((8, 2, 136), F16, 1), draw((8, 2, 136), F16, 1), docs),
        lambda: L.attend(q, k, k[:4], docs),                                             # other rows
        lambda: L.attend(q.cpu(), k, k, docs),
        lambda: L.attend(q.transpose(1, 2), k, k, docs),
        lambda: L.attend(draw((8, 4, 68), F16, 1)[:, :, 4:], k, k, docs),                # not aligned
        lambda: L.attend(q, k, k, docs, cap=-1.0),
        lambda: L.attend(q, k, k, docs, cap=math.nan),
        lambda: L.attend(q, k, k, docs, scale=math.inf),
        lambda: L.attend(q, k, k, docs, slopes=torch.ones(3, device="cuda")),
        lambda: L.attend(q, k, k, docs, slopes=torch.ones(4, dtype=F16, device="cuda")),
        lambda: L.attend(q, k, k, L.Documents(o, o), slopes=torch.ones(4, device="cuda")),        # slopes without positions
        lambda: L.attend(q[:6], k, k, docs),                                             # positions of other rows
        lambda: L.Documents(o.long(), o),
        lambda: L.Documents(o, o[:2]),
        lambda: L.Documents(o, o, k_lens=o),
        lambda: L.Documents(o.cpu(), o.cpu()),
        lambda: L.attend(q, k, k, L.Documents(o[:1], o[:1])),                            # rows without documents
        lambda: L.attend_backward(q[:, :2], q, k, k, q, torch.zeros(8, 4, device="cuda"), docs),
        lambda: L.attend_backward(q, q, k, k, q, torch.zeros(8, 2, device="cuda"), docs),
        lambda: L.norm_rotate(q, k[:4], w, w),
        lambda: L.norm_rotate(q, k, w[:32], w),
        lambda: L.norm_rotate(q, k, w.half(), w),
        lambda: L.norm_rotate(q, k, w, w, table=L.rotation_table(8, 32)),                # a table without positions
        lambda: L.norm_rotate(q, k, w, w, pos=o, table=L.rotation_table(8, 32)),
        lambda: L.norm_rotate(q, k, w, w, pos=torch.zeros(8, dtype=torch.int32, device="cuda"), table=torch.zeros(8, 24, device="cuda")),
        lambda: L.norm_rotate(q, k, w, w, pos=torch.zeros(8, dtype=torch.int32, device="cuda"), table=torch.zeros(8, 80, device="cuda")),
        lambda: L.norm_rotate(q, k, w, w, eps=-1.0),
        lambda: L.norm_rotate(draw((8, 1, 264), F16, 1), draw((8, 1, 264), F16, 1), draw((264,), F32, 1), draw((264,), F32, 1)),
        lambda: L.rotation_table(0, 32),
        lambda: L.rotation_table(5, 24),
        lambda: L.pack_activations(q),
        lambda: L.pack_activations(torch.zeros(4, 4, dtype=torch.int8, device="cuda")),
        lambda: L.pack_activations(torch.zeros(4, 8, device="cuda").t()),
        lambda: L.pack_activations(torch.zeros(4, 8)),
        lambda: L.pack_activations(torch.zeros(4, 8, device="cuda"), pos=o),
        lambda: L.packed_weight_grad(L.pack_activations(torch.zeros(4, 8, device="cuda")), torch.zeros(4, 8, dtype=F16, device="cuda")),
        lambda: L.packed_weight_grad(L.pack_activations(torch.zeros(4, 8, dtype=F16, device="cuda")), torch.zeros(3, 8, dtype=F16, device="cuda")),
        lambda: L.packed_weight_grad(L.pack_activations(torch.zeros(4, 8, dtype=F16, device="cuda")), torch.zeros(4, 8, device="cuda")),
        lambda: L.PackedActivations(torch.zeros(4, 8, dtype=torch.int8, device="cuda"), torch.zeros(4, 1, dtype=torch.uint8, device="cuda"), 8, F16),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(L.LegionPrepError):
            f()
            pytest.fail(f"call {i} was taken")
