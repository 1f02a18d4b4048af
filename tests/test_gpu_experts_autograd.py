"""The routed expert products and autograd: gradients are calls of their own, so
a loss that is differentiated through a result raises instead of leaving the
inputs without gradients; results keep their values, and an autograd function
around the calls works."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

T, E, K, N, D = 40, 6, 2, 72, 64


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def rand(shape, dtype, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * scale).to(dtype)


def calls(g):
    """(name, inputs that may want a gradient, call of them giving tensors)."""
    logits, x, w = rand((T, E), torch.float32, 1), rand((T, D), torch.bfloat16, 2), rand((E, N, D), torch.bfloat16, 3)
    r = g.route(logits, K)
    y = rand((T * K, N), torch.bfloat16, 4)
    q, s = g.quantise_blocks(x)
    wq, ws = g.quantise_blocks(w, 128)
    return [
        ("route", [logits], lambda l: [g.route(l, K).weight, g.route(l, K).group_weight]),
        ("group_product", [x, w], lambda a, b: [g.group_product(a, b, r.group_ptr, index=r.token)]),
        ("combine", [y, r.weight], lambda a, b: [g.combine(a, r.row_ptr, r.slot, b)]),
        ("quantise_blocks", [x], lambda a: list(g.quantise_blocks(a))),
        ("group_product_fp8", [s, ws], lambda a, b: [g.group_product_fp8(q, a, wq, b, r.group_ptr, index=r.token)]),
    ]


def test_differentiating_raises_and_values_stay(g):
    for name, inputs, call in calls(g):
        want = call(*inputs)
        assert not any(t.requires_grad for t in want)
        for i in range(len(inputs)):
            given = [t.detach().clone().requires_grad_(j == i) for j, t in enumerate(inputs)]
            got = call(*given)
            for a, b in zip(want, got):
                assert torch.equal(a.float(), b.detach().float()), name
                with pytest.raises(RuntimeError, match="gmagnus.%s has no autograd formula" % name):
                    b.float().sum().backward()
            assert given[i].grad is None
            with torch.no_grad():
                assert not any(t.requires_grad for t in call(*given)), name


def test_results_can_be_changed_in_place_and_out_has_no_graph(g):
    x, w = rand((T, D), torch.bfloat16, 2), torch.nn.Parameter(rand((E, N, D), torch.bfloat16, 3))
    r = g.route(rand((T, E), torch.float32, 1), K)
    y = g.group_product(x, w, r.group_ptr, index=r.token)
    y += 1
    buf = torch.empty((T * K, N + 8), dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        out = g.group_product(x, w, r.group_ptr, index=r.token, out=buf[:, 8:])
        assert not out.requires_grad and not buf.requires_grad
    assert torch.equal(out + 1, y.detach())
    # gradients made by hand are not part of a graph
    d = g.group_outer(y.detach(), x.clone().requires_grad_(), r.group_ptr, index=r.token)
    assert not d.requires_grad


def test_inside_an_autograd_function(g):
    class Product(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, group_ptr):
            ctx.save_for_backward(x, w, group_ptr)
            return g.group_product(x, w, group_ptr)

        @staticmethod
        def backward(ctx, d_y):
            x, w, group_ptr = ctx.saved_tensors
            return g.group_product(d_y, w, group_ptr, transposed=True), g.group_outer(d_y, x, group_ptr), None

    gp = torch.tensor([0, 10, 10, 40], device="cuda")
    x = rand((40, D), torch.bfloat16, 1).requires_grad_()
    w = rand((3, N, D), torch.bfloat16, 2).requires_grad_()
    d_y = rand((40, N), torch.bfloat16, 3)
    Product.apply(x, w, gp).backward(d_y)
    d, xs, ws = d_y.double(), x.detach().double(), w.detach().double()
    for e, (b, f) in enumerate(((0, 10), (10, 10), (10, 40))):
        for got, want, mag in ((x.grad[b:f], d[b:f] @ ws[e], d[b:f].abs() @ ws[e].abs()),
                               (w.grad[e], d[b:f].t() @ xs[b:f], d[b:f].abs().t() @ xs[b:f].abs())):
            assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 100 * 2.0 ** -23 * mag).all())
