"""The operators together: a gated layer with its norm, trained and served. Gradients against a plain 64-bit layer
(autograd), serving in every form against it, the whole step as a graph."""
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
    spec = importlib.util.spec_from_file_location("gated_expert_layer", os.path.join(ROOT, "examples", "gated_expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


SIZES = [(50, 6, 2, 64, 96), (1, 4, 1, 40, 24), (33, 5, 3, 65, 130), (64, 16, 4, 256, 128)]


def case(ex, tokens, experts, k, hidden, inner):
    gen = torch.Generator(device="cuda").manual_seed(3)
    layer = ex.GatedExpertLayer(hidden, inner, experts, k, gen)
    x, residual, d_out, d_total = (torch.randn(tokens, hidden, device="cuda", generator=gen).bfloat16() for _ in range(4))
    return layer, x, residual, d_out, d_total


def plain(layer, x, residual, chosen, eps):
    """The layer in 64 bits on the host with a given choice of experts, as leaves and results."""
    leaves = [v.double().cpu().requires_grad_() for v in (x, residual, layer.norm, layer.router, layer.w1, layer.w2)]
    x, residual, norm, router, w1, w2 = leaves
    h = x + residual
    y = h * (h.square().mean(1, keepdim=True) + eps).rsqrt() * norm
    p = torch.softmax((y @ router).masked_fill(~chosen, -float("inf")), 1)
    gate, up = torch.matmul(y, w1.transpose(1, 2)).chunk(2, 2)
    out = torch.matmul(gate * torch.sigmoid(gate) * up, w2.transpose(1, 2))  # experts x tokens x hidden
    return leaves, (p.t()[:, :, None] * out).sum(0), h


def choice(r):
    chosen = torch.zeros(r.n_tokens, r.n_experts, dtype=torch.bool)
    rows = torch.repeat_interleave(torch.arange(r.n_tokens), (r.row_ptr[1:] - r.row_ptr[:-1]).cpu())
    chosen[rows, r.expert[:len(rows)].cpu().long()] = True
    return chosen


def off(a, b):
    return float((a.double().cpu() - b).norm() / b.norm().clamp(min=1e-12))


@pytest.mark.parametrize("tokens,experts,k,hidden,inner", SIZES)
def test_gradients(ex, tokens, experts, k, hidden, inner):
    layer, x, residual, d_out, d_total = case(ex, tokens, experts, k, hidden, inner)
    out, total, saved = layer.forward(x, residual)
    got = layer.backward(d_out, d_total, saved)
    leaves, want, h = plain(layer, x, residual, choice(saved[2]), ex.EPS)
    (want * d_out.double().cpu()).sum().add((h * d_total.double().cpu()).sum()).backward()
    # every step rounds to bfloat16 (2^-8 relative): the sum, the norm, the product, the gate (of a product of two), the
    # product and the sum on the way to the result; six more on the longest way back
    assert off(out, want.detach()) <= 7 * 2.0 ** -8 and off(total, h.detach()) <= 2.0 ** -8
    dx, dnorm, drouter, dw1, dw2 = got
    for a, b in ((dx, leaves[0].grad), (dx, leaves[1].grad), (dnorm, leaves[2].grad), (drouter, leaves[3].grad), (dw1, leaves[4].grad),
                 (dw2, leaves[5].grad)):
        assert off(a, b) <= 13 * 2.0 ** -8 or float(b.norm()) < 1e-9


@pytest.mark.parametrize("tokens,experts,k,hidden,inner", SIZES)
def test_serving_forms(ex, tokens, experts, k, hidden, inner):
    layer, x, residual, _, _ = case(ex, tokens, experts, k, hidden, inner)
    saved = layer.forward(x, residual)[2]
    _, want, _ = plain(layer, x, residual, choice(saved[2]), ex.EPS)
    want = want.detach()
    fp8, int8 = layer.quantised(torch.float8_e4m3fn), layer.quantised(torch.int8)
    # (the logits are the same in all forms, so the choice is)
    assert off(layer.serve(x, residual)[0], want) <= 7 * 2.0 ** -8
    assert off(layer.serve_few(x, residual)[0], want) <= 4 * 2.0 ** -8      # the sum, the norm, the result (and the logits' rows)
    # values of E4M3 are off by 2^-4 at most, 2^-4 / sqrt(3) a value as they come: rows, W1, gate, W2 and the two halves of a product
    assert off(layer.serve_few(x, residual, fp8)[0], want) <= 4 * 2.0 ** -4
    assert off(layer.serve(x, residual, fp8)[0], want) <= 6 * 2.0 ** -4
    assert off(layer.serve_few(x, residual, int8)[0], want) <= 3 * 4 / 254 + 4 * 2.0 ** -8  # (weights: W1 twice, W2)
    # integers: half a step is 1 / 254 of a row's largest, four times its mean square root at most here
    assert off(layer.serve(x, residual, int8)[0], want) <= 6 * 4 / 254 + 7 * 2.0 ** -8


def test_a_step_and_a_served_batch_as_graphs(ex):
    layer, x, residual, d_out, d_total = case(ex, 48, 8, 2, 128, 96)
    int8 = layer.quantised(torch.int8)

    def work():
        out, total, saved = layer.forward(x, residual)
        return (out, total) + layer.backward(d_out, d_total, saved) + layer.serve(x, residual, int8) + layer.serve_few(x, residual)

    work()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for turn in range(4):
        gen = torch.Generator(device="cuda").manual_seed(20 + turn)
        for t in (x, residual, d_out):
            t.copy_(torch.randn(t.shape, device="cuda", generator=gen))
        want = [t.clone() for t in work()]
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_example_runs(ex):
    r = ex.main(["--tokens", "256", "--experts", "8", "--hidden", "128", "--inner", "128", "--steps", "3"])
    assert r["few"] <= 10 * 2.0 ** -8 and len(r["losses"]) == 3 and all(v == v for v in r["losses"])
