"""The routed expert products at the sizes that their inner loops run over in real
use (experts_cases.py; which kernel each case takes is looked at without a GPU in
test_experts_launches.py), and at offsets past 32 bits of every operand. Against
64-bit forms on the GPU, group by group; bounds as in test_gpu_experts_tiles.py."""
import numpy as np
import pytest

from tests import experts_cases as ec
from tests import experts_ref as er

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

B, H, F = "bfloat16", "float16", "float32"


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


def offsets(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int64).cuda()


def picks(n, rows, seed):
    return torch.randint(0, n, (rows,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def within(y, want, mag, terms, dtype, more=0.0):
    limit = er.U[dtype] * want.abs() + er.TINY[dtype] + (terms + 8) * 2.0 ** -23 * mag + more
    assert bool(((y.double() - want).abs() <= limit).all())


def adder(r, m):
    """What the matrix units may lose on E4M3 operands: 16 products are aligned to their largest and cut 13 bits below its
    leading bit."""
    r, m = (torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 16)).unflatten(1, (-1, 16)).amax(2) for v in (r, m.t()))
    return 2.0 ** -9 * (r @ m.t().contiguous())


@pytest.mark.parametrize("kernel,sizes,n,k,transposed", ec.PRODUCTS)
@pytest.mark.parametrize("dtype,out", [(B, B), (H, H), (B, F), (H, F)])
@pytest.mark.parametrize("gather", [True, False])
def test_products(g, kernel, sizes, n, k, transposed, dtype, out, gather):
    rows, gp = sum(sizes), offsets(sizes)
    # (an index into half as many rows; rows of their own without one)
    n_x = max(1, rows // 2) if gather else rows
    index = picks(n_x, rows, 3) if gather else None
    t, o = getattr(torch, dtype), getattr(torch, out)
    x, w = rand((n_x, k), t, 1), rand((len(sizes),) + ((k, n) if transposed else (n, k)), t, 2, k ** -0.5)
    y = g.group_product(x, w, gp, index=index, transposed=transposed, out=torch.full((rows, n), float("nan"), dtype=o, device="cuda"))
    b = gp.tolist()
    for e, size in enumerate(sizes):
        if size:
            r = (x[index[b[e]:b[e + 1]].long()] if gather else x[b[e]:b[e + 1]]).double()
            m = w[e].double() if transposed else w[e].double().t().contiguous()
            within(y[b[e]:b[e + 1]], r @ m, r.abs() @ m.abs(), k, out)


@pytest.mark.parametrize("kernel,sizes,n,k", ec.FP8_PRODUCTS)
@pytest.mark.parametrize("out", [B, H, F])
@pytest.mark.parametrize("gather", [True, False])
def test_fp8_products(g, kernel, sizes, n, k, out, gather):
    rows, gp = sum(sizes), offsets(sizes)
    n_x = max(1, rows // 2) if gather else rows
    index = picks(n_x, rows, 3) if gather else None
    # every block of a row and of the weights has a scale of its own size
    x = rand((n_x, k), torch.float32, 1) * torch.exp2(rand((n_x, -(-k // 128)), torch.float32, 4))[:, torch.arange(k, device="cuda") // 128]
    w = rand((len(sizes), n, k), torch.float32, 2, k ** -0.5)
    w *= torch.exp2(rand((len(sizes), 1, -(-k // 128)), torch.float32, 5))[:, :, torch.arange(k, device="cuda") // 128]
    q, s = g.quantise_blocks(x)
    wq, ws = g.quantise_blocks(w, 128)
    y = g.group_product_fp8(q, s, wq, ws, gp, index=index,
                            out=torch.full((rows, n), float("nan"), dtype=getattr(torch, out), device="cuda"))
    up, down = torch.arange(k, device="cuda") // 128, torch.arange(n, device="cuda") // 128
    xv = q.double() * s.double()[:, up]
    b = gp.tolist()
    for e, size in enumerate(sizes):
        if size:
            r = xv[index[b[e]:b[e + 1]].long()] if gather else xv[b[e]:b[e + 1]]
            m = (wq[e].double() * ws[e].double()[down][:, up]).t().contiguous()
            within(y[b[e]:b[e + 1]], r @ m, r.abs() @ m.abs(), k, out, adder(r, m))


@pytest.mark.parametrize("kernel,by_size,sizes,n,k", ec.OUTERS)
@pytest.mark.parametrize("dtype,out", [(B, B), (H, F)])
@pytest.mark.parametrize("gather", [True, False])
def test_outers(g, kernel, by_size, sizes, n, k, dtype, out, gather):
    rows, gp = sum(sizes), offsets(sizes)
    n_x = max(1, rows // 2) if gather else rows
    t, o = getattr(torch, dtype), getattr(torch, out)
    x, d_y = rand((n_x, k), t, 1), rand((rows, n), t, 2)
    index = picks(n_x, rows, 3) if gather else None
    d = g.group_outer(d_y, x, gp, index=index, out=torch.full((len(sizes), n, k), float("nan"), dtype=o, device="cuda"))
    b = gp.tolist()
    for e, size in enumerate(sizes):
        r = (x[index[b[e]:b[e + 1]].long()] if gather else x[b[e]:b[e + 1]]).double()
        m = d_y[b[e]:b[e + 1]].double().t().contiguous()
        within(d[e], m @ r, m.abs() @ r.abs(), size, out)


@pytest.mark.parametrize("k", [1, 127, 1920, 2048, 2049, 2176, 3969, 4096, 4100, 6144, 8192, 8320, 12289])
@pytest.mark.parametrize("dtype", [B, H, F])
def test_quantise_long_rows(g, k, dtype):
    # a work group takes 16 blocks of 128 at a time, two of them in flight: 16, 32 and more blocks a row, and what is left
    x = rand((37, k), getattr(torch, dtype), k) * torch.exp2(rand((37, -(-k // 128)), torch.float32, 1))[
        :, torch.arange(k, device="cuda") // 128].to(getattr(torch, dtype))
    for v in (x, torch.stack([x, x.flip(0)])):
        q, s = g.quantise_blocks(v)
        h = v.float().cpu()
        b = torch.nn.functional.pad(h, (0, -k % 128)).unflatten(-1, (-1, 128))
        want_s = np.maximum(b.abs().amax(-1).numpy() / np.float32(448), np.float32(2.0 ** -126))
        assert np.array_equal(s.cpu().numpy(), want_s)
        want_q = np.clip(h.numpy() / er.spread_scale(want_s, 1, 37, k), -448, 448)
        assert torch.equal(q.cpu().view(torch.uint8), torch.from_numpy(want_q).to(torch.float8_e4m3fn).view(torch.uint8))


# ------------------------------------------------------- offsets past 32 bits
def far_rows(n_rows, n, dtype):
    """Rows of n elements, so far apart that the last ones lie past 4 GiB."""
    stride = (1 << 32) // n_rows // dtype.itemsize + 4096
    return torch.empty((n_rows, stride), dtype=dtype, device="cuda")[:, 8:8 + n]


@pytest.mark.parametrize("n,k,transposed", [(136, 64, False), (136, 64, True), (45, 67, False), (40, 61, True)])
@pytest.mark.parametrize("out", [B, F])
def test_results_past_32_bits(g, n, k, transposed, out):
    # Y's rows reach past 4 GiB: in a tall group, in a few rows of the last groups and in the zeros past them
    sizes = [4096 - 40, 3, 17]
    rows = sum(sizes) + 20
    y = far_rows(rows, n, getattr(torch, out))
    assert (rows - 1) * y.stride(0) * y.element_size() > 1 << 32
    y.fill_(float("nan"))
    x, w = rand((rows, k), torch.bfloat16, 1), rand((3,) + ((k, n) if transposed else (n, k)), torch.bfloat16, 2, k ** -0.5)
    gp = offsets(sizes)
    g.group_product(x, w, gp, transposed=transposed, out=y)
    b = gp.tolist()
    for e in range(3):
        r, m = x[b[e]:b[e + 1]].double(), w[e].double() if transposed else w[e].double().t().contiguous()
        within(y[b[e]:b[e + 1]], r @ m, r.abs() @ m.abs(), k, out)
    assert not y[b[-1]:].any()


def far_stack(e, n, k, dtype):
    """A stack of matrices so far apart that the last one lies past 4 GiB."""
    size = torch.empty(0, dtype=dtype).element_size()
    apart = ((1 << 32) // (e - 1) // size + n * k) // 128 * 128
    return torch.empty((e - 1) * apart + n * k, dtype=dtype, device="cuda").as_strided((e, n, k), (apart, k, 1))


@pytest.mark.parametrize("n,k", [(72, 1096), (264, 136), (33, 77)])
@pytest.mark.parametrize("rows", [4, 40, 100])
def test_weights_and_their_gradients_past_32_bits(g, n, k, rows):
    e = 3
    gp = offsets([rows] * e)
    w = far_stack(e, n, k, torch.bfloat16)
    for i in range(e):
        w[i] = rand((n, k), torch.bfloat16, i)
    x, d_y = rand((e * rows, k), torch.bfloat16, 7), rand((e * rows, n), torch.bfloat16, 8)
    y, d_x = g.group_product(x, w, gp), g.group_product(d_y, w, gp, transposed=True)
    for i in range(e):
        r, m, d = x[i * rows:(i + 1) * rows].double(), w[i].double(), d_y[i * rows:(i + 1) * rows].double()
        within(y[i * rows:(i + 1) * rows], r @ m.t().contiguous(), r.abs() @ m.t().abs().contiguous(), k, B)
        within(d_x[i * rows:(i + 1) * rows], d @ m, d.abs() @ m.abs(), n, B)
    out = w.fill_(float("nan"))
    g.group_outer(d_y, x, gp, out=out)
    for i in range(e):
        d, r = d_y[i * rows:(i + 1) * rows].double().t().contiguous(), x[i * rows:(i + 1) * rows].double()
        within(out[i], d @ r, d.abs() @ r.abs(), rows, B)


@pytest.mark.parametrize("n,k", [(136, 2064), (45, 300)])
@pytest.mark.parametrize("rows", [4, 40, 100])
def test_fp8_weights_and_rows_past_32_bits(g, n, k, rows):
    e = 3
    gp = offsets([rows] * e)
    wq = far_stack(e, n, k, torch.float8_e4m3fn)
    v, ws = g.quantise_blocks(rand((e, n, k), torch.float32, 1), 128)
    wq.view(torch.uint8).copy_(v.view(torch.uint8))
    x = rand((e * rows, k), torch.bfloat16, 2)
    a, s = g.quantise_blocks(x)
    want = g.group_product_fp8(a, s, v, ws, gp)
    assert torch.equal(g.group_product_fp8(a, s, wq, ws, gp), want)
    del wq
    # rows of X past 4 GiB take the tiles for any alignment: sums in another order
    q = far_rows(e * rows, k, torch.float8_e4m3fn)
    q.view(torch.uint8).copy_(a.view(torch.uint8))
    y = g.group_product_fp8(q, s, v, ws, gp, index=torch.arange(e * rows, dtype=torch.int32, device="cuda"))
    up, down = torch.arange(k, device="cuda") // 128, torch.arange(n, device="cuda") // 128
    xv = a.double() * s.double()[:, up]
    for i in range(e):
        r, m = xv[i * rows:(i + 1) * rows], (v[i].double() * ws[i].double()[down][:, up]).t().contiguous()
        within(y[i * rows:(i + 1) * rows], r @ m, r.abs() @ m.abs(), k, B, adder(r, m))


def test_combine_past_32_bits(g):
    t, k, n = 300, 2, 40
    r = g.route(rand((t, 8), torch.float32, 1), k)
    y, out = far_rows(t * k, n, torch.bfloat16), far_rows(t, n, torch.bfloat16)
    y.copy_(rand((t * k, n), torch.bfloat16, 2))
    near = y.contiguous()
    g.combine(y, r.row_ptr, r.slot, r.weight, out=out)
    assert torch.equal(out, g.combine(near, r.row_ptr, r.slot, r.weight))
    d_out = out.copy_(rand((t, n), torch.bfloat16, 3))
    got = g.combine_backward(y, r.row_ptr, r.slot, r.weight, d_out)
    for a, b in zip(got, g.combine_backward(near, r.row_ptr, r.slot, r.weight, d_out.contiguous())):
        assert torch.equal(a, b)
