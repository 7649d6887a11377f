"""Derivatives that the operators do not compute are refused (no GPU needed)."""
import pytest
import torch


@pytest.mark.parametrize("op", ["add_norm", "gated_linear", "attend", "norm_rotate"])
def test_forward_mode_derivatives_are_refused(op):
    """A tangent needs no gradient, and the kernels would read the values and lose it.  Refused before anything else is looked at, so tensors of the CPU show it."""
    import torch.autograd.forward_ad as forward

    import paper_2305_16588_amd as L
    x, w, one = torch.ones(4, 8), torch.ones(3, 8), torch.ones(4, 2, 8)
    calls = dict(add_norm=lambda t: [lambda: L.add_norm(t(x), x, w[0]), lambda: L.add_norm(x, t(x), w[0]), lambda: L.add_norm(x, None, t(w[0]))],
                 gated_linear=lambda t: [lambda: L.gated_linear(t(x), w, w), lambda: L.gated_linear(x, t(w), w), lambda: L.gated_linear(x, w, t(w))],
                 attend=lambda t: [lambda: L.attend(t(one), one, one, None), lambda: L.attend(one, t(one), one, None), lambda: L.attend(one, one, t(one), None),
                                   lambda: L.attend(one, one, one, None, slopes=t(w[0, :2]))],
                 norm_rotate=lambda t: [lambda: L.norm_rotate(t(one), one, x[0], x[0]), lambda: L.norm_rotate(one, t(one), x[0], x[0]),
                                        lambda: L.norm_rotate(one, one, t(x[0]), x[0]), lambda: L.norm_rotate(one, one, x[0], t(x[0]))])[op]
    for leaf in (False, True):
        with forward.dual_level():
            for call in calls(lambda t: forward.make_dual(t.clone().requires_grad_(leaf), torch.ones_like(t))):
                with pytest.raises(L.LegionPrepError, match="forward-mode"):
                    call()
