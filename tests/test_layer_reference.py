"""The 64-bit definitions that the operators of a model layer are tested against, against differences (no GPU needed); the C entry points' own refusals."""
import ctypes as C

import torch

import layer_common as ref


def difference(f, x, h=1e-5):
    """Gradient of the scalar f by every element of x, by central differences."""
    g = torch.zeros_like(x)
    flat, out = x.view(-1), g.view(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        out[i] = (up - f()) / (2 * h)
        flat[i] = keep
    return g


def test_attention_gradients_are_the_differences(monkeypatch):
    monkeypatch.setitem(ref.UNIT, torch.float64, 0.0)
    monkeypatch.setitem(ref.TINY, torch.float64, 0.0)
    torch.manual_seed(1)
    for cap, bias in ((0.0, False), (1.5, True)):
        q, k, v, w = (torch.randn(s, dtype=torch.float64) for s in ((5, 4, 8), (7, 2, 8), (7, 2, 8), (5, 4, 8)))
        slopes = torch.rand(4, dtype=torch.float64) if bias else None
        docs = dict(spans=[(0, 2, 0, 3), (2, 1, 3, 0), (3, 2, 3, 3)], q_pos=torch.tensor([0, 1, 2, 0, 3]), k_pos=torch.tensor([0, 2, 1, 0, 5, 1, 1]))

        def loss():
            return float((ref.attention(q, k, v, docs, None, slopes, cap)["out"][0] * w).sum())

        got = ref.attention(q, k, v, docs, w, slopes, cap)
        for x, name in ((q, "dq"), (k, "dk"), (v, "dv")) + (((slopes, "d_slopes"),) if bias else ()):
            assert torch.allclose(got[name][0], difference(loss, x), atol=1e-8), name
        assert (got["out"][0][2] == 0).all() and (got["lse"][0][2] == -float("inf")).all() and (got["dk"][0][6] == 0).all()


def test_norm_gradients_are_the_differences(monkeypatch):
    monkeypatch.setitem(ref.UNIT, torch.float64, 0.0)
    torch.manual_seed(2)
    x, w, g = torch.randn(4, 2, 16, dtype=torch.float64), torch.randn(16, dtype=torch.float64), torch.randn(4, 2, 16, dtype=torch.float64)
    pos = torch.tensor([3, -1, 0, 4])
    angle = torch.arange(5, dtype=torch.float64)[:, None] * torch.rand(4, dtype=torch.float64)
    table = torch.cat([angle.cos(), angle.sin()], 1)

    def loss():
        return float((ref.head_norm(x, w, pos, table, 1e-5)["out"][0] * g).sum())

    got = ref.head_norm(x, w, pos, table, 1e-5, g)
    assert torch.allclose(got["dx"][0], difference(loss, x), atol=1e-8)
    assert torch.allclose(got["dw"][0], difference(loss, w), atol=1e-8)


def test_packed_values_are_near_and_of_the_type():
    torch.manual_seed(3)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        x = (torch.randn(20, 70) * torch.exp2(torch.randint(-30, 12, (20, 1)).float())).to(dtype)
        values, exps, held = ref.pack(x)
        assert torch.equal(held, held.to(dtype).double())
        for g in range(0, 70, 32):
            part, top = x[:, g:g + 32].double(), x[:, g:g + 32].double().abs().amax(1, keepdim=True)
            least = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -127
            # half a step, or a whole one for what lies within the last half step below a power of two
            assert ((part - held[:, g:g + 32]).abs() <= torch.maximum(top / 64, torch.full_like(top, least))).all()


def test_c_entry_points_refuse_what_makes_no_sense():
    import paper_2305_16588_amd as lgp
    b, L = lgp.binding, lgp.load_library()
    size, p = C.c_size_t(7), 4096          # an aligned address that is never read

    def docs(**kw):
        a = dict(n_docs=1, q_rows=8, k_rows=8, q_offsets=p, k_offsets=p, q_lens=None, k_lens=None, q_pos=p, k_pos=p)
        return b._Documents(*{**a, **kw}.values())

    def att(**kw):
        a = dict(q=p, k=p, v=p, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, heads=4, kv_heads=2, dim=64, dtype=1, scale=0.125, cap=0.0, slopes=None)
        return b._Attention(*{**a, **kw}.values())

    def forward(d, a, out=p, lse=p):
        return L.lgp_attend(0, C.byref(d) if d else None, C.byref(a) if a else None, out, None, lse, None, 0, None)

    assert forward(None, att()) == -1 and forward(docs(), None) == -1
    for kw in (dict(n_docs=-1), dict(n_docs=0), dict(q_rows=-1), dict(q_offsets=None), dict(k_offsets=None)):
        assert forward(docs(**kw), att()) == -1, kw
    for kw in (dict(q=None), dict(v=None), dict(k=p + 8), dict(heads=3), dict(kv_heads=0), dict(dim=0), dict(q_row=4), dict(v_head=12), dict(cap=-1.0),
               dict(cap=float("nan")), dict(scale=float("inf"))):
        assert forward(docs(), att(**kw)) == -1, kw
    for kw in (dict(dtype=0), dict(dtype=3), dict(dim=12), dict(dim=136)):
        assert forward(docs(), att(**kw)) == -4, kw
    assert forward(docs(q_rows=2 ** 30), att()) == -4 and forward(docs(k_rows=2 ** 31), att()) == -4
    assert forward(docs(q_pos=None), att(slopes=p)) == -1
    assert forward(docs(), att(), out=None) == -1 and forward(docs(), att(), lse=None) == -1 and forward(docs(), att(), out=p + 2) == -1
    assert L.lgp_attend_workspace(0, C.byref(docs()), C.byref(att()), 0, None) == -1
    assert L.lgp_attend_backward(0, C.byref(docs()), C.byref(att()), p, p, None, p, None, p, p, None, p, 1 << 20, None) == -1
    assert L.lgp_attend_backward(0, C.byref(docs()), C.byref(att()), p, p, None, p, p, p, p, p, p, 1 << 20, None) == -1       # slopes' gradient without slopes

    def heads(**kw):
        a = dict(q=p, k=p, q_row=256, q_head=64, k_row=128, k_head=64, tokens=8, heads=4, kv_heads=2, dim=64, dtype=0, q_weight=p, k_weight=p, pos=p, rot=32, n_pos=9,
                 table=p, eps=1e-6)
        return b._Heads(*{**a, **kw}.values())

    for kw in (dict(q=None), dict(tokens=-1), dict(heads=0, kv_heads=0), dict(q_weight=None), dict(table=None), dict(pos=None), dict(n_pos=0), dict(rot=80),
               dict(q_row=12), dict(k=p + 4), dict(eps=-1.0)):
        assert L.lgp_norm_rotate(0, C.byref(heads(**kw)), p, p, None) == -1, kw
    for kw in (dict(dtype=5), dict(dim=20, rot=0), dict(dim=264), dict(rot=24)):
        assert L.lgp_norm_rotate(0, C.byref(heads(**kw)), p, p, None) == -4, kw
    assert L.lgp_norm_rotate(0, C.byref(heads()), None, p, None) == -1
    assert L.lgp_norm_rotate_workspace(0, C.byref(heads()), None) == -1
    assert L.lgp_norm_rotate_backward(0, C.byref(heads()), p, p, p, p, None, p, p, 1 << 20, None) == -1

    def packed(**kw):
        return b._Packed(*{**dict(tokens=8, width=40, dtype=1, values=p, exps=p, pos=None), **kw}.values())

    for kw in (dict(tokens=-1), dict(width=0), dict(values=None), dict(exps=None), dict(values=p + 8)):
        assert L.lgp_pack_activations(0, p, 40, C.byref(packed(**kw)), None) == -1, kw
    assert L.lgp_pack_activations(0, p, 40, C.byref(packed(dtype=9)), None) == -4 and L.lgp_pack_activations(0, None, 40, C.byref(packed()), None) == -1
    assert L.lgp_unpack_activations(0, C.byref(packed()), None, None) == -1
    assert L.lgp_packed_weight_grad_workspace(0, C.byref(packed()), 0, C.byref(size)) == -1 and size.value == 0
    assert L.lgp_packed_weight_grad(0, C.byref(packed()), p, 8, 1, 8, None, None, None, 0, None) == -1
    assert L.lgp_packed_weight_grad(0, C.byref(packed(dtype=0)), p, 8, 1, 8, p, None, None, 0, None) == -4                    # fp16 from a wider range
    assert L.lgp_packed_weight_grad(0, C.byref(packed()), p, 8, 0, 8, p, None, None, 0, None) == -4
