"""The gate where sigma is below fp32's normal numbers and its product with g and u is not, and its gradient where
products on the way pass fp32's largest number: relative errors as anywhere else."""
import pytest

from tests import rows_ref as rr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def near(got, want, error, dtype):
    """As the results' type rounds; beyond its largest value anything of that sign."""
    got = got.double().cpu()
    top = torch.finfo(dtype).max
    ok = (got - want).abs() <= rr.half_step(dtype) * (want.abs() + error) + error + rr.TINY[dtype]
    return bool((ok | ((want.abs() + error > top) & (got.sign() == want.sign()) & (got.abs() >= top / 2))).all())


def far_rows(dtype):
    """A row for every u: g from -60 to -210, and some around it."""
    gate = torch.cat((torch.linspace(-210, -60, 601), torch.linspace(-87.5, -85.5, 101), torch.tensor([-1e4, -3e38, 5.0, 60.0, 90.0, 3e30])))
    up = torch.tensor([2.0 ** e * s for e in (-120, -60, 0, 1, 60, 100, 120, 126) for s in (1.0, -1.7)])
    g, u = torch.meshgrid(gate, up, indexing="xy")
    return g.to(dtype), u.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [707, 704, 40, 4])
def test_gate(g, dtype, n):
    a, u = far_rows(dtype)
    for c in range(0, a.shape[1] - n + 1, n):
        h = torch.cat((a[:, c:c + n], u[:, c:c + n]), 1)
        want = rr.gate(h)
        # e^g 8 units, three products and a rounding
        assert near(g.gate(h.cuda()).y, want, 12 * rr.U32 * want.abs(), dtype)
    wide = torch.cat((a.repeat(1, 24), u.repeat(1, 24)), 1)  # (rows that are read in passes)
    want = rr.gate(wide)
    assert near(g.gate(wide.cuda()).y, want, 12 * rr.U32 * want.abs(), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [707, 704])
def test_gate_backward(g, dtype, n):
    a, u = (t[:, :n] for t in far_rows(dtype))
    for e in (-100, -30, 0, 40, 100, 125):
        d = torch.full_like(a, 1.3 * 2.0 ** e)
        h = torch.cat((a, u), 1)
        want, mag = rr.gate_backward(h, d)
        # five more operations; a product below fp32's normal numbers loses half a subnormal's step
        assert near(g.gate_backward(h.cuda(), d.cuda()), want, 20 * rr.U32 * mag + 2.0 ** -149, dtype)
    # near the slope's zero, with products beyond fp32 on the way
    a = torch.linspace(-1.4, -1.1, 64).repeat(3, 1).to(dtype)
    u, d = torch.full_like(a, 2.0 ** 100), torch.full_like(a, 2.0 ** 40)
    h = torch.cat((a, u), 1)
    want, mag = rr.gate_backward(h, d)
    assert near(g.gate_backward(h.cuda(), d.cuda()), want, 20 * rr.U32 * mag, dtype)


@pytest.mark.parametrize("tokens", [1, 20])
def test_expert_layer(g, tokens):
    # products of one term: g and u are the weights; W2 takes each gate's result alone
    f = 130
    gate = torch.linspace(-130, -84, f).bfloat16()
    x = torch.ones((tokens, 1), dtype=torch.bfloat16).cuda()
    w2 = torch.eye(f, dtype=torch.bfloat16)[None].cuda()
    for e in (60, 90, 120):
        u = torch.full_like(gate, 2.0 ** e)
        w1 = torch.cat((gate, u))[None, :, None].cuda()
        y = g.expert_layer(x, torch.zeros((tokens, 1), device="cuda"), 1, w1, w2, out_dtype=torch.float32)
        want = rr.gate(torch.cat((gate, u))[None])
        # two values of the rows' type (of which the smaller may be below its normal numbers)
        off = (12 * rr.U32 + rr.half_step(torch.bfloat16) ** 2) * want.abs() + rr.TINY[torch.bfloat16]
        assert bool(((y.double().cpu() - want).abs() <= off + rr.U32 * want.abs()).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [8, 77, 1032, 20001])
def test_values_do_not_change_with_what_lies_beside_them(g, dtype, n):
    gen = torch.Generator().manual_seed(n)
    rows = 300 if n < 5000 else 5
    h, d = (torch.randn((rows, k), generator=gen).mul_(3).to(dtype).cuda() for k in (2 * n, n))
    h[0, :n // 2 + 1] = 1e-30 if dtype != torch.float16 else 1e-7  # (products that may end below normal numbers)
    d[0] *= 1e-3
    y, back = g.gate(h).y, g.gate_backward(h, d)
    other = h.clone()
    places = torch.rand((rows, n), generator=gen).cuda() < 0.05
    places[:, 0] = True
    other[:, :n][places] = -100.0
    if dtype != torch.float16:
        d = d.clone()
        d[:, n - 1], other[:, 2 * n - 1] = 1e30, 1e30
        places[:, n - 1] = True
    y2, back2 = g.gate(other).y, g.gate_backward(other, d)
    keep = ~places
    assert torch.equal(y[keep], y2[keep])
    assert torch.equal(back[:, :n][keep], back2[:, :n][keep]) and torch.equal(back[:, n:][keep], back2[:, n:][keep])
