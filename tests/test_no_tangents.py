"""Forward-mode differentiation: a call whose operand has a tangent raises (before anything else is looked at, so
without a GPU too), instead of giving results without one."""
import pytest

torch = pytest.importorskip("torch")
gm = pytest.importorskip("paper_2607_22866_amd.gmagnus")
fw = torch.autograd.forward_ad

CALLS = [
    ("rms_norm", lambda t: gm.rms_norm(t)), ("rms_norm", lambda t: gm.rms_norm(t.detach(), residual=t)),
    ("rms_norm_backward", lambda t: gm.rms_norm_backward(t.detach(), None, t)), ("gate", lambda t: gm.gate(t)),
    ("gate_backward", lambda t: gm.gate_backward(t.detach(), t)), ("quantise_rows", lambda t: gm.quantise_rows(t)),
    ("expert_layer", lambda t: gm.expert_layer(t, t.detach(), 1, t.detach(), t.detach())),
    ("group_product", lambda t: gm.group_product(t.detach(), t, t.detach())), ("combine", lambda t: gm.combine(t, t, t)),
    ("route", lambda t: gm.route(t, 1)), ("quantise_blocks", lambda t: gm.quantise_blocks(t)),
    ("group_product_int8", lambda t: gm.group_product_int8(t.detach(), t, t.detach(), t.detach(), t.detach())),
]


@pytest.mark.parametrize("name,call", CALLS)
def test_tangents_raise(name, call):
    x = torch.ones(4, 8)
    with fw.dual_level():
        with pytest.raises(RuntimeError, match="gmagnus.%s has no formula for forward-mode" % name):
            call(fw.make_dual(x, torch.ones_like(x)))
        with pytest.raises(ValueError, match="CUDA tensor"):  # (no tangent: as ever)
            call(x)
    with pytest.raises(ValueError, match="CUDA tensor"):
        call(x)


def test_routing_with_a_tangent():
    n = torch.zeros(2)
    with fw.dual_level():
        w = fw.make_dual(n, n + 1)
        r = gm.Routing(1, 2, 2, True, n, n, w, n, n, n, n)
        with pytest.raises(RuntimeError, match="route_backward has no formula for forward-mode"):
            gm.route_backward(n, r, n)
