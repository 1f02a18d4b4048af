"""Gradients of the norm and of the gate that are differentiated once more raise, instead of counting as constants."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def test_second_derivatives_raise(g):
    inputs = [rand((6, 40), torch.bfloat16, 1), rand((40,), torch.bfloat16, 2), rand((6, 40), torch.bfloat16, 3), rand((6, 40), torch.bfloat16, 4)]
    calls = [("rms_norm_backward", lambda h, w, d, t: g.rms_norm_backward(h, w, d, d_total=t), inputs),
             ("gate_backward", lambda h, d: (g.gate_backward(h, d),), [inputs[0], rand((6, 20), torch.bfloat16, 5)])]
    for name, call, given in calls:
        want = call(*given)
        assert not any(t.requires_grad for t in want)
        for i in range(len(given)):
            args = [t.clone().requires_grad_(j == i) for j, t in enumerate(given)]
            for a, b in zip(want, call(*args)):
                assert torch.equal(a, b.detach())
                with pytest.raises(RuntimeError, match="gmagnus.%s has no autograd formula" % name):
                    b.float().sum().backward()
            with torch.no_grad():
                assert not any(t.requires_grad for t in call(*args))
    out = torch.empty((6, 40), dtype=torch.bfloat16, device="cuda")
    assert not g.gate_backward(inputs[0].clone().requires_grad_(), inputs[2][:, :20], out=out).requires_grad
    d_x, d_w = g.rms_norm_backward(inputs[0].clone().requires_grad_(), None, inputs[2])
    assert d_w is None and d_x.requires_grad


def test_gradient_of_a_gradient_inside_an_autograd_function(g):
    class Gate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h):
            ctx.save_for_backward(h)
            return g.gate(h).y

        @staticmethod
        def backward(ctx, d):
            h, = ctx.saved_tensors
            return g.gate_backward(h, d)

    h = rand((5, 32), torch.float32, 7).requires_grad_()
    d = rand((5, 16), torch.float32, 8)
    once, = torch.autograd.grad(Gate.apply(h), h, d)
    assert torch.equal(once, g.gate_backward(h.detach(), d))
    twice, = torch.autograd.grad(Gate.apply(h), h, d, create_graph=True)
    with pytest.raises(RuntimeError, match="gate_backward has no autograd formula"):
        twice.sum().backward()
