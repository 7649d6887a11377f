"""The 64-bit definitions of what a layer has around its attention, against differences (no GPU needed); the C entry points' own refusals."""
import ctypes as C
import math

import torch

import dense_common as ref
import layer_common
from test_layer_reference import difference


def exact(monkeypatch):
    for of in (layer_common.UNIT, layer_common.TINY):
        monkeypatch.setitem(of, torch.float64, 0.0)


def test_norm_gradients_are_the_differences(monkeypatch):
    exact(monkeypatch)
    torch.manual_seed(1)
    x, res, a, b = (torch.randn(5, 12, dtype=torch.float64) for _ in range(4))
    w, pos = torch.randn(12, dtype=torch.float64), torch.tensor([3, -1, 0, 4, -7])

    def loss():
        r = ref.add_norm(x, res, w, pos, 1e-3)
        return float((r["y"][0] * a).sum() + (r["total"] * b).sum())

    total = ref.add_norm(x, res, w, pos, 1e-3)["total"]
    assert torch.equal(total[1], torch.zeros(12, dtype=torch.float64)) and torch.equal(total[0], x[0] + res[0])
    got = ref.add_norm(None, None, w, pos, 1e-3, a, torch.where(pos[:, None] >= 0, b, 0.0), total)
    for t, name in ((x, "dx"), (res, "d_residual"), (w, "dw")):
        assert torch.allclose(got[name][0], difference(loss, t), atol=1e-8), name


def test_gated_gradients_are_the_differences(monkeypatch):
    exact(monkeypatch)
    torch.manual_seed(2)
    x, g, u, a = (torch.randn(s, dtype=torch.float64) for s in ((6, 8), (5, 8), (5, 8), (6, 5)))
    pos = torch.tensor([0, 1, -1, 2, 3, -4])
    for act in ("silu", "gelu"):
        def loss():
            return float((ref.gated(x, g, u, act, pos)["h"][0] * a).sum())

        got = ref.gated(x, g, u, act, pos, a)
        for t, name in ((x, "dx"), (g, "dw_gate"), (u, "dw_up")):
            assert torch.allclose(got[name][0], difference(loss, t), atol=1e-8), (act, name)
        plain = torch.nn.functional.silu if act == "silu" else torch.nn.functional.gelu
        assert torch.allclose(got["h"][0][pos >= 0], (plain(x @ g.T) * (x @ u.T))[pos >= 0], atol=1e-12) and (got["h"][0][pos < 0] == 0).all()


def test_clipping_of_the_definition():
    grads = [torch.tensor([3.0, 0.0]), torch.tensor([[4.0]]), torch.zeros(0)]
    norm, out = ref.clip(grads, 1.0)
    assert norm == 5.0 and torch.allclose(out[0], torch.tensor([0.6, 0.0], dtype=torch.float64)) and float(out[1]) == 0.8
    assert ref.clip(grads, 10.0)[1][0][0] == 3.0 and ref.clip([torch.zeros(3)], 1.0)[0] == 0.0
    assert ref.clip([torch.tensor([math.inf])], 1.0)[1][0][0] == math.inf


def test_c_entry_points_refuse_what_makes_no_sense():
    import paper_2305_16588_amd as lgp
    b, L = lgp.binding, lgp.load_library()
    size, p = C.c_size_t(7), 4096          # an aligned address that is never read

    def residual(**kw):
        a = dict(x=p, residual=p, x_row=40, residual_row=40, tokens=8, width=40, dtype=2, stream_dtype=0, weight=p, pos=p, eps=1e-6)
        return C.byref(b._Residual(*{**a, **kw}.values()))

    def rows(**kw):
        return C.byref(b._Rows8(*{**dict(tokens=8, width=40, values=p, scales=p, pos=None), **kw}.values()))

    for kw in (dict(tokens=-1), dict(width=0), dict(x=None), dict(weight=None), dict(weight=p + 2), dict(eps=-1.0), dict(eps=float("nan")), dict(residual=None)):
        assert L.lgp_add_norm(0, residual(**kw), p, p, None) == -1, kw
        assert L.lgp_add_norm_rows8(0, residual(**kw), rows(), p, None) == -1, kw
    for kw in (dict(dtype=7), dict(stream_dtype=1), dict(width=16385), dict(tokens=2 ** 33), dict(dtype=0, stream_dtype=2)):
        assert L.lgp_add_norm(0, residual(**kw), p, p, None) == -4, kw
    assert L.lgp_add_norm(0, None, p, p, None) == -1 and L.lgp_add_norm(0, residual(), None, p, None) == -1 and L.lgp_add_norm(0, residual(), p, None, None) == -1
    for kw in (dict(tokens=7), dict(width=41), dict(values=None), dict(scales=None), dict(values=p + 8)):
        assert L.lgp_add_norm_rows8(0, residual(), rows(**kw), p, None) == -1, kw
    assert L.lgp_add_norm_workspace(0, residual(), None) == -1 and L.lgp_add_norm_workspace(0, residual(width=0), C.byref(size)) == -1 and size.value == 0
    back = dict(dy=p, d_total=p, dx=p, d_residual=p, d_weight=p, workspace=p, size=1 << 20)

    def backward(r, **kw):
        a = {**back, **kw}
        return L.lgp_add_norm_backward(0, r, a["dy"], a["d_total"], a["dx"], a["d_residual"], a["d_weight"], a["workspace"], a["size"], None)

    for kw in (dict(dy=None), dict(dx=None), dict(d_residual=None), dict(d_weight=None)):
        assert backward(residual(), **kw) == -1, kw
    assert backward(residual(dtype=0)) == -1                      # one type: one gradient
    assert backward(residual(residual=None)) == -1
    assert L.lgp_pack_rows8(0, None, 40, 0, rows(), None) == -1 and L.lgp_pack_rows8(0, p, 40, 5, rows(), None) == -4 and L.lgp_pack_rows8(0, p, 40, 0, rows(width=16385), None) == -4

    def product(r, w, out=p, dtype=0):
        return L.lgp_linear_rows8(0, r, w, None, dtype, out, None)

    assert product(None, rows()) == -1 and product(rows(), None) == -1 and product(rows(), rows(width=41)) == -1 and product(rows(), rows(tokens=0)) == -1
    assert product(rows(), rows(), None) == -1 and product(rows(values=p + 4), rows()) == -1 and product(rows(), rows(scales=None)) == -1
    assert product(rows(), rows(), p, 9) == -4 and product(rows(width=(1 << 17) + 1), rows(width=(1 << 17) + 1)) == -4 and product(rows(tokens=(1 << 24) + 1), rows()) == -4

    def gated(**kw):
        a = dict(x=p, x_row=40, tokens=8, width=40, hidden=24, dtype=1, act=0, w_gate=p, w_up=p, pos=p)
        return C.byref(b._Gated(*{**a, **kw}.values()))

    for kw in (dict(x=None), dict(tokens=-1), dict(width=0), dict(hidden=0), dict(w_gate=None), dict(w_up=p + 8), dict(x=p + 2), dict(x_row=44), dict(x_row=-8), dict(x_row=1 << 22)):
        assert L.lgp_gated_linear(0, gated(**kw), p, None, 0, None) == -1, kw
        assert L.lgp_gated_linear_workspace(0, gated(**kw), 1, C.byref(size)) == -1, kw
    for kw in (dict(dtype=0), dict(act=2), dict(width=44), dict(width=65544), dict(hidden=65537), dict(tokens=(1 << 24) + 1)):
        assert L.lgp_gated_linear(0, gated(**kw), p, None, 0, None) == -4, kw
    assert L.lgp_gated_linear(0, gated(), None, None, 0, None) == -1 and L.lgp_gated_linear_workspace(0, gated(), 0, None) == -1
    assert L.lgp_gated_linear_workspace(0, gated(), 0, C.byref(size)) == 0 and size.value == 0
    assert L.lgp_gated_linear_workspace(0, gated(tokens=5000), 0, C.byref(size)) == 0 and size.value >= 20_000       # a list of its tokens
    assert L.lgp_gated_linear_workspace(0, gated(), 1, C.byref(size)) == 0 and size.value >= 8 * 2 * 64 * 2
    for kw in ((None, p, p, p), (p, None, p, p), (p, p, None, p), (p, p, p, None), (p, p + 8, p, p)):
        assert L.lgp_gated_linear_backward(0, gated(), *kw, p, 1 << 20, None) == -1, kw

    def gradients(*of):
        return (b._Gradient * len(of))(*(b._Gradient(*g) for g in of))

    def clip(of, most=1.0, norm=p, n=None):
        return L.lgp_clip_gradients(0, of, len(of) if n is None else n, most, norm, p, 1 << 20, None)

    one = (p, p, 10, 0)
    assert clip(gradients(one), -1.0) == -1 and clip(gradients(one), float("nan")) == -1 and clip(gradients(one), 1.0, None) == -1 and clip(gradients(one), n=-1) == -1
    assert L.lgp_clip_gradients(0, None, 1, 1.0, p, p, 1 << 20, None) == -1
    for g in ((None, p, 10, 0), (p, None, 10, 0), (p, p, -1, 0), (p + 2, p + 2, 10, 0), (p + 1, p + 1, 10, 1)):
        assert clip(gradients(g)) == -1, g
    assert clip(gradients((p, p, 10, 3))) == -4 and clip(gradients((p, p, 1 << 38, 0))) == -4 and clip(gradients(one), n=65537) == -4
    # written ranges that overlap: the same twice, one that reaches into the next, results over another's gradient, results over each other
    q = p + 4096
    for of in ((one, one), (one, (p + 36, p + 36, 4, 0)), ((p, q, 10, 0), (q + 8, q + 8, 2, 0)), ((p, q, 10, 0), (p + 64, q + 39, 1, 0)), ((p, p + 4, 10, 0),)):
        assert clip(gradients(*of)) == -1, of
    assert L.lgp_clip_gradients_workspace(0, None) == -1
