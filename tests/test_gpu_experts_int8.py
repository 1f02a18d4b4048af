"""Grouped products of 8-bit integers on the GPU: their sums are exact, so a result is a few roundings off at most
(the sum as fp32, two products, the result's type)."""
import numpy as np
import pytest

from tests import experts_ref as er
from tests import int8_cases as ic

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def integers(shape, seed, low=-127):
    return torch.randint(low, 128, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int8).cuda()


def scales(shape, seed):
    return (torch.rand(shape, generator=torch.Generator().manual_seed(seed)) + 0.1).cuda() * 0.01


def offsets(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int64).cuda()


def reference(x, xs, w, ws, gp, index, n_rows):
    """64-bit results on the GPU (integer products below 2^53 are exact there)."""
    rows = torch.arange(n_rows, device="cuda") if index is None else index.long()
    there = (rows >= 0) & (rows < x.shape[0])
    xv = torch.where(there[:, None], x.double()[rows.clamp(0, x.shape[0] - 1)], 0.0)
    sv = torch.where(there, xs.double()[rows.clamp(0, x.shape[0] - 1)], 0.0)
    y = torch.zeros(n_rows, w.shape[1], dtype=torch.float64, device="cuda")
    for e in range(len(gp) - 1):
        b, f = min(max(gp[e], 0), n_rows), min(gp[e + 1], n_rows)
        if b < f:
            y[b:f] = (xv[b:f] @ w[e].double().t()) * sv[b:f, None] * ws[e].double()[None]
    return y


def check(g, x, xs, w, ws, sizes, index=None, extra=0, out_dtype=torch.bfloat16, gp=None):
    gp = offsets(sizes) if gp is None else gp
    n_rows = x.shape[0] if index is None else index.numel()
    out = torch.full((n_rows, w.shape[1]), float("nan"), dtype=out_dtype, device="cuda")
    y = g.group_product_int8(x, xs, w, ws, gp, index=index, out_dtype=out_dtype, out=out)
    want = reference(x, xs, w, ws, gp.tolist(), index, n_rows)
    name = str(out_dtype).replace("torch.", "")
    # the sum as fp32, times x's scale, times w's: three roundings, then the result's
    off = want.abs() * (er.U[name] + 3.01 * 2.0 ** -24) + er.TINY[name]
    assert bool(((y.double() - want).abs() <= off).all())
    return y


@pytest.mark.parametrize("kernel,sizes,n,k", ic.PRODUCTS)
def test_every_kernel(g, kernel, sizes, n, k):
    rows = sum(sizes)
    x, w = integers((rows, k), 1), integers((len(sizes), n, k), 2)
    index = torch.randint(0, rows, (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    for out_dtype in (torch.bfloat16, torch.float16, torch.float32):
        check(g, x, scales((rows,), 4), w, scales((len(sizes), n), 5), sizes, index=index, out_dtype=out_dtype)
    check(g, x, scales((rows,), 4), w, scales((len(sizes), n), 5), sizes, out_dtype=torch.float32)


@pytest.mark.parametrize("n,k", [(1, 1), (1, 127), (5, 128), (16, 129), (64, 16), (130, 257), (33, 1040), (257, 300)])
@pytest.mark.parametrize("sizes", [[1], [3, 0, 17, 1], [0, 0, 0], [16, 128, 15, 129, 0, 64], [300, 5]])
def test_sizes(g, n, k, sizes):
    rows = sum(sizes) + 3
    x, w = integers((rows, k), n), integers((len(sizes), n, k), k)
    y = check(g, x, scales((rows,), 4), w, scales((len(sizes), n), 5), sizes)
    assert not y[sum(sizes):].any()  # rows of no group
    index = torch.randint(-2, rows + 2, (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    check(g, x, scales((rows,), 4), w, scales((len(sizes), n), 5), sizes, index=index, out_dtype=torch.float32)


@pytest.mark.parametrize("rows", [2, 40, 300])
@pytest.mark.parametrize("k", [2048, 2050])
def test_sums_are_exact_to_the_ends(g, rows, k):
    # the largest sums: -128 * -128 in every place, and sums that cancel but for one
    x = torch.full((rows, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((1, 96, k), -128, dtype=torch.int8, device="cuda")
    w[0, 1::2, ::2] = 127
    w[0, 1::2, 1::2] = -127
    w[0, 3, 5] = -126
    one, ones = torch.ones(rows, device="cuda"), torch.ones((1, 96), device="cuda")
    y = g.group_product_int8(x, one, w, ones, offsets([rows]), out_dtype=torch.float32)
    want = (x.double() @ w[0].double().t())
    assert torch.equal(y.double(), want) and float(want[0, 3]) == -128.0


def test_longest_rows(g):
    k = 131071
    x = torch.full((3, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((1, 20, k), -128, dtype=torch.int8, device="cuda")
    y = g.group_product_int8(x, torch.ones(3, device="cuda"), w, torch.ones((1, 20), device="cuda"), offsets([3]), out_dtype=torch.float32)
    assert bool((y == float(np.float32(128 * 128 * k))).all())
    with pytest.raises(g.GmagnusError) as e:
        g.group_product_int8(integers((3, k + 1), 1), torch.ones(3, device="cuda"), integers((1, 20, k + 1), 2),
                             torch.ones((1, 20), device="cuda"), offsets([3]))
    assert e.value.status == 6


def test_rows_as_quantise_rows_gives_them(g):
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn((50, 200), generator=gen).bfloat16().cuda(), torch.randn((4, 72, 200), generator=gen).cuda()
    (q, s), (wq, ws) = g.quantise_rows(x), g.quantise_rows(w)
    y = check(g, q, s, wq, ws, [10, 0, 25, 15], out_dtype=torch.float32)
    # every value is off by at most half its row's scale, so a sum of products x w by at most the sum of
    # |x| sw / 2 + |w| sx / 2 + sx sw / 4 (and the result's own roundings)
    for e, b, f in ((0, 0, 10), (2, 10, 35), (3, 35, 50)):
        xe, we, sx, sw = x[b:f].double(), w[e].double(), s[b:f].double()[:, None], ws[e].double()[None]
        off = xe.abs().sum(1, keepdim=True) * sw / 2 + we.abs().sum(1)[None] * sx / 2 + 200 * sx * sw / 4
        full = xe @ we.t()
        assert bool(((y[b:f].double() - full).abs() <= off + 4 * 2.0 ** -24 * (full.abs() + off)).all())


def test_strides_and_alignment(g):
    sizes = [20, 0, 31]
    xw, ww = integers((51, 700), 1), integers((3, 80, 700), 2)
    sx, sw = scales((51,), 3), scales((3, 200), 4)
    for off, k, n in ((0, 640, 80), (1, 640, 77), (16, 333, 80), (5, 512, 64)):
        x, w, ws = xw[:, off:off + k], ww[:, :n, off:off + k], sw[:, off:off + n]
        a = check(g, x, sx, w, ws, sizes, out_dtype=torch.float32)
        b = g.group_product_int8(x.contiguous(), sx, w.contiguous(), ws.contiguous(), offsets(sizes), out_dtype=torch.float32)
        assert torch.equal(a, b)
        buf = torch.full((51, n + 9), 5.0, device="cuda")
        g.group_product_int8(x, sx, w, ws, offsets(sizes), out=buf[:, 4:4 + n])
        assert torch.equal(buf[:, 4:4 + n], a) and bool((buf[:, :4] == 5).all()) and bool((buf[:, 4 + n:] == 5).all())


def test_part_of_the_groups_and_bounds_beyond_the_rows(g):
    x, w = integers((40, 256), 1), integers((3, 48, 256), 2)
    sx, sw = scales((40,), 3), scales((3, 48), 4)
    for gp in ([5, 20, 20, 33], [-7, 3, 10, 900], [40, 40, 40, 40]):
        t = torch.tensor(gp, dtype=torch.int64, device="cuda")
        check(g, x, sx, w, sw, None, gp=t, out_dtype=torch.float32)


def test_offsets_past_31_bits(g):
    # rows of X beyond 2 GiB, and an operand as wide
    n_x, k = (1 << 20) + 40, 2064
    x = torch.zeros((n_x, k), dtype=torch.int8, device="cuda")
    last = integers((40, k), 1)
    x[-40:] = last
    w, sw = integers((1, 64, k), 2), scales((1, 64), 3)
    sx = scales((n_x,), 4)
    index = torch.arange(n_x - 40, n_x, dtype=torch.int32, device="cuda")
    y = g.group_product_int8(x, sx, w, sw, offsets([40]), index=index, out_dtype=torch.float32)
    assert torch.equal(y, g.group_product_int8(last, sx[-40:], w, sw, offsets([40]), out_dtype=torch.float32))


def test_graph_and_stream(g):
    x, w = integers((64, 512), 1), integers((4, 128, 512), 2)
    sx, sw, gp = scales((64,), 3), scales((4, 128), 4), offsets([16] * 4)
    want = g.group_product_int8(x, sx, w, sw, gp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = g.group_product_int8(x, sx, w, sw, gp, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = g.group_product_int8(x, sx, w, sw, gp)
    for turn in range(3):
        x.copy_(integers((64, 512), 10 + turn))
        want = g.group_product_int8(x, sx, w, sw, gp)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_rows_and_refusals(g):
    w, sw = integers((2, 16, 32), 1), scales((2, 16), 2)
    gp = offsets([0, 0])
    x = integers((0, 32), 3)
    assert g.group_product_int8(x, torch.ones(0, device="cuda"), w, sw, gp).shape == (0, 16)
    x, sx = integers((4, 32), 3), scales((4,), 4)
    y = g.group_product_int8(x, sx, w, sw, gp)
    assert y.shape == (4, 16) and not y.any()
    for call in (lambda: g.group_product_int8(x.float(), sx, w, sw, gp), lambda: g.group_product_int8(x, sx[:3], w, sw, gp),
                 lambda: g.group_product_int8(x, sx.half(), w, sw, gp), lambda: g.group_product_int8(x, sx, w[0], sw, gp),
                 lambda: g.group_product_int8(x, sx, w, sw[:1], gp), lambda: g.group_product(x, w, gp)):
        with pytest.raises((ValueError, g.GmagnusError)):
            call()
    with pytest.raises(RuntimeError, match="group_product_int8 has no autograd formula"):
        g.group_product_int8(x, sx.clone().requires_grad_(), w, sw, gp).float().sum().backward()
