"""The operators of a model layer together, as the example uses them: its gradients against automatic differentiation in 64 bits, and a training
that learns; documents that the single-query kernels meet with several queries or none."""
import math

import pytest
import torch

import layer_common as ref
from test_gpu_9_layer import BF16, F16, draw, lgp, make_docs, run_attention

pytestmark = pytest.mark.gpu


def test_gradients_of_the_layer():
    """Relative error of every gradient in the 2-norm.  Activations in 8 bits are 0.7 % off (a step is a 64th to a 128th of the largest of 32), at random
    over the tokens that a gradient is summed over; each of about ten roundings to bf16 between them 0.2 %: together less than 2 %."""
    L = lgp()
    from paper_2305_16588_amd.example_layer import AttentionLayer, Neighbourhoods
    g = torch.Generator().manual_seed(3)
    n, fanout, width, H, D = 300, 10, 100, 4, 32
    cnt = torch.randint(0, fanout + 1, (n,), generator=g, dtype=torch.int32).cuda()
    nbr = torch.randint(0, 5000, (n, fanout), generator=g, dtype=torch.int32).cuda()
    nbr[torch.arange(fanout, device="cuda") >= cnt[:, None]] = -1
    hoods = Neighbourhoods(torch.arange(n, dtype=torch.int32, device="cuda"), nbr, cnt)
    x = draw((n * (1 + fanout), width), torch.float32, 5).bfloat16()
    target = draw((n,), torch.float32, 6)
    layer = AttentionLayer(width, H, D, seed=7)
    layer.w["qkv_bias"] += draw((3 * H * D,), torch.float32, 8, 0.1)
    loss, got = layer.step(torch.where((hoods.pos >= 0)[:, None], x, math.nan), hoods, target)

    w = {k: t.double().requires_grad_() for k, t in layer.w.items()}
    live = hoods.pos >= 0
    X = torch.where(live[:, None], x.double(), 0.0)
    qkv = (X @ w["qkv"].t() + w["qkv_bias"]).view(-1, 3 * H, D)

    def norm(t, weight):
        t = t / torch.sqrt((t * t).mean(2, keepdim=True) + 1e-6) * weight
        turn = layer.table[hoods.pos.clamp(min=0).long()].double()[:, None]
        half = layer.table.shape[1] // 2
        c, s, a, b = turn[..., :half], turn[..., half:], t[..., :half], t[..., half:2 * half]
        return torch.cat([a * c - b * s, b * c + a * s, t[..., 2 * half:]], 2)

    rows = 1 + fanout
    q, k, v = (t.view(n, rows, H, D).transpose(1, 2) for t in (norm(qkv[:, :H], w["q_norm"]), norm(qkv[:, H:2 * H], w["k_norm"]), qkv[:, 2 * H:]))
    z = layer.cap * torch.tanh(q @ k.transpose(2, 3) * D ** -0.5 / layer.cap)
    p = hoods.pos.view(n, rows)
    z = z - w["slopes"][None, :, None, None] * (p[:, None, :, None] - p[:, None, None, :]).abs().double()
    z = z.masked_fill(~live.view(n, 1, 1, rows), -math.inf)
    out = (torch.softmax(z, 3) @ v)[:, :, 0].reshape(n, H * D)
    want = ((out @ w["out"] - target.double()) ** 2).mean()
    want.backward()
    assert abs(float(loss) / float(want.detach()) - 1) < 0.01
    for name, t in w.items():
        off = float((got[name].double() - t.grad).norm() / t.grad.norm())
        assert off < 0.02, f"{name}: {off:.4f}"


def test_the_example_learns():
    from paper_2305_16588_amd import example_layer
    losses = example_layer.main(["--steps", "40"])
    assert all(math.isfinite(x) for x in losses) and sum(losses[-5:]) < 0.5 * sum(losses[:5])


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [(F16, 32, 4, 4), (BF16, 64, 4, 2), (F16, 16, 2, 1), (BF16, 128, 70, 70)])
@pytest.mark.parametrize("q_owned,q_tokens", [([1] * 12, None), ([0, 3, 0, 1, 0, 0, 2, 1, 1, 0, 1, 3], None), ([1] * 12, [0, 1, 1, 0, 1, 1, 1, 1, 1, 0, 1, 1]),
                                              ([12] + [0] * 11, None)])
def test_documents_of_one_query_on_average(q_owned, q_tokens, dtype, dim, heads, kv_heads):
    keys = [5, 0, 64, 1, 17, 3, 40, 2, 16, 9, 0, 33]
    docs, info = make_docs(q_owned, keys, q_tokens)
    run_attention(docs, info, heads, kv_heads, dim, dtype, 20.0, True)
    run_attention(docs, info, heads, kv_heads, dim, dtype, scale=-0.2)
    docs, info = make_docs(q_owned, [k + 3 for k in keys], q_tokens, keys)
    run_attention(docs, info, heads, kv_heads, dim, dtype, 0.0, True, rest=False)


@pytest.mark.parametrize("heads,kv_heads", [(3, 1), (10, 2), (7, 7), (16, 1), (32, 1), (48, 2)])
def test_groups_of_every_kind(heads, kv_heads):
    """Heads that share a key head: as many as are folded into rows of a tile, and numbers that are not."""
    docs, info = make_docs([40, 1, 7, 100], [30, 60, 7, 100])
    run_attention(docs, info, heads, kv_heads, 64, BF16, 0.0, True)
    docs, info = make_docs([1, 1, 2], [600, 3, 2000])
    run_attention(docs, info, heads, kv_heads, 32, F16, 0.0, False)


@pytest.mark.parametrize("order", [1, -1])
def test_capped_scores_near_and_far(order):
    """Both ways to the tanh, in one tile and in tiles of their own; scores that grow and fall from tile to tile, so that their base is raised."""
    docs, info = make_docs([70], [400])
    L = lgp()
    q, k, v, g = draw((70, 2, 64), BF16, 1), draw((400, 2, 64), BF16, 2), draw((400, 2, 64), BF16, 3), draw((70, 2, 64), BF16, 4)
    size = torch.linspace(0.05, 12, 400, device="cuda")
    size = size if order > 0 else size.flip(0)
    k = (k.float() * size[:, None, None]).bfloat16()
    for cap in (5.0, 0.0):
        out, lse, rest = L.attend(q, k, v, docs, cap=cap, rest=True)
        got = L.attend_backward(g, q, k, v, out, lse, docs, rest=rest, cap=cap)
        want = ref.attention(q, k, v, info, g, None, cap)
        for x, name in zip((out, lse, *got[:3]), ("out", "lse", "dq", "dk", "dv")):
            ref.check(x, want[name], f"{name}, cap {cap}")


def test_documents_far_from_where_they_are_looked_for():
    """Lengths so uneven that a tile's document is none of those around where it would be if all were alike."""
    owned = [0] * 300 + [900] + [1] * 300 + [0] * 200 + [700, 64, 33]
    docs, info = make_docs(owned, owned)
    run_attention(docs, info, 2, 1, 32, F16, 0.0, True)
    docs, info = make_docs(owned[::-1], owned)
    run_attention(docs, info, 2, 2, 64, BF16)


def test_strides_that_are_too_large_are_refused():
    L = lgp()
    docs, _ = make_docs([2], [2])
    q = torch.empty(1 << 25, dtype=F16, device="cuda").as_strided((2, 1, 64), (1 << 24, 64, 1))
    with pytest.raises(L.LegionPrepError):
        L.attend(q, q, q, docs)
