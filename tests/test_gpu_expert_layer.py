"""The example layer of experts: its gradients against a plain float32 layer
(autograd), its training, its serving by single tokens and in 8 bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens,experts,k,hidden,inner", [(50, 6, 2, 64, 96), (1, 4, 1, 40, 24), (33, 5, 3, 65, 130)])
def test_gradients(ex, tokens, experts, k, hidden, inner):
    gen = torch.Generator(device="cuda").manual_seed(3)
    layer = ex.ExpertLayer(hidden, inner, experts, k, gen)
    x = torch.randn(tokens, hidden, device="cuda", generator=gen).bfloat16()
    d_out = torch.randn(tokens, hidden, device="cuda", generator=gen).bfloat16()
    out, saved = layer.forward(x)
    got = layer.backward(d_out, saved)
    xs, router, w1, w2 = (v.double().cpu().requires_grad_() for v in (x, layer.router, layer.w1, layer.w2))
    logits = xs @ router
    chosen = torch.zeros(tokens, experts, dtype=torch.bool)
    r = saved[2]
    rows = torch.repeat_interleave(torch.arange(tokens), (r.row_ptr[1:] - r.row_ptr[:-1]).cpu())
    chosen[rows, r.expert.cpu().long()] = True
    p = torch.softmax(logits.masked_fill(~chosen, -float("inf")), 1)
    h = torch.nn.functional.silu(torch.matmul(xs, w1.transpose(1, 2)))  # experts x tokens x inner
    y = torch.matmul(h, w2.transpose(1, 2))
    want = (p.t()[:, :, None] * y).sum(0)
    want.backward(d_out.double().cpu())
    # every step rounds to bfloat16 (2^-8 relative); the longest way to a gradient has seven such steps
    assert float((out.double().cpu() - want.detach()).norm() / want.detach().norm()) <= 4 * 2.0 ** -8
    for a, b in zip(got, (xs.grad, router.grad, w1.grad, w2.grad)):
        assert float((a.double().cpu() - b).norm() / b.norm().clamp(min=1e-12)) <= 7 * 2.0 ** -8 or float(b.norm()) < 1e-9


def test_example_runs(ex):
    r = ex.main(["--tokens", "512", "--experts", "8", "--hidden", "128", "--inner", "256", "--steps", "20"])
    assert r["losses"][-1] < 0.9 * r["losses"][0]
    assert r["one"] <= 2.0 ** -7      # (sums in another order, rounded to bfloat16)
    assert r["eight"] <= 0.1          # (two products of operands rounded to 2^-4 each, averaged)
    assert int(r["together"].diagonal().sum()) == 512 * 2
