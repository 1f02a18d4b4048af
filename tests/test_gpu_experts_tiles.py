"""The grouped products at sizes that reach the largest tiles (groups of 384 rows
and more, enough of them to fill the card), with groups that end at, before and
behind a tile's edges and half tiles' edges; and the low and high rows a group
may have between the kernels' limits. Bounds as in test_gpu_experts.py, for
8-bit operands from how the matrix units add; the 64-bit references are formed on the GPU, group by group."""
import numpy as np
import pytest

from tests import experts_ref as er

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# 16 groups, 8192 rows: 0, 1, one below / at / above 128 and 256, and long ones
EDGES = [0, 1, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511, 640, 1000, 1600, 2136]


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


def within(y, want, mag, terms, dtype, more=0.0):
    name = str(dtype).replace("torch.", "")
    limit = er.U[name] * want.abs() + er.TINY[name] + (terms + 8) * 2.0 ** -23 * mag + more
    assert bool(((y.double() - want).abs() <= limit).all())


def check_product(g, sizes, n, k, dtype, transposed, gather, out_dtype=None, extra=0):
    rows = sum(sizes) + extra
    gp = offsets(sizes)
    n_x = rows // 3 if gather else rows
    index = torch.randint(0, n_x, (rows,), dtype=torch.int32, device="cuda",
                          generator=torch.Generator(device="cuda").manual_seed(n + k)) if gather else None
    x = rand((n_x, k), dtype, 1)
    w = rand((len(sizes),) + ((k, n) if transposed else (n, k)), dtype, 2, k ** -0.5)
    y = g.group_product(x, w, gp, index=index, transposed=transposed, out_dtype=out_dtype,
                        out=torch.full((rows, n), float("nan"), dtype=out_dtype or dtype, device="cuda"))
    b = gp.tolist()
    for e, size in enumerate(sizes):
        if size:
            r = x[index[b[e]:b[e + 1]].long()].double() if gather else x[b[e]:b[e + 1]].double()
            m = w[e].double() if transposed else w[e].double().t().contiguous()
            within(y[b[e]:b[e + 1]], r @ m, r.abs() @ m.abs(), k, out_dtype or dtype)
    assert not y[b[-1]:].any()


@pytest.mark.parametrize("n,k", [(1536, 8), (1536, 64), (1544, 72), (1536, 200), (1800, 136)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("transposed", [False, True])
def test_large_tiles(g, n, k, dtype, transposed):
    check_product(g, EDGES, n, k, dtype, transposed, gather=not transposed, extra=70)


@pytest.mark.parametrize("transposed", [False, True])
def test_large_tiles_other_order_and_type(g, transposed):
    check_product(g, EDGES[::-1], 1536, 328, torch.bfloat16, transposed, gather=transposed, out_dtype=torch.float32)
    check_product(g, [4096], 4096, 192, torch.float16, transposed, gather=False)


@pytest.mark.parametrize("mean", [16, 17, 40, 41, 96, 97, 200])
@pytest.mark.parametrize("transposed", [False, True])
def test_every_tile_height(g, mean, transposed):
    # means of rows a group on both sides of the kernels' limits, sizes spread around them
    sizes = [0, 2 * mean, mean // 2, mean + mean - mean // 2, mean - 1, mean + 1]
    for n, k in ((4096 if mean == 16 else 328, 264), (130, 72), (135, 97)):
        check_product(g, sizes, n, k, torch.bfloat16, transposed, gather=True, extra=3)


@pytest.mark.parametrize("n,k", [(1024, 768), (1000, 776), (392, 2048)])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_large_tiles_outer(g, n, k, gather, dtype):
    # 70 groups: more than the 64 that are ordered by size together
    sizes = (EDGES + [3, 64, 65, 0, 700] + [5] * 49) if n == 392 else EDGES
    rows = sum(sizes) + 11
    gp = offsets(sizes)
    n_x = rows // 2 if gather else rows
    index = torch.randint(-1, n_x + 1, (rows,), dtype=torch.int32, device="cuda") if gather else None
    x, d_y = rand((n_x, k), dtype, 1), rand((rows, n), dtype, 2)
    d = g.group_outer(d_y, x, gp, index=index)
    b = gp.tolist()
    for e, size in enumerate(sizes):
        if gather:
            ids = index[b[e]:b[e + 1]].long()
            r = torch.where(((ids >= 0) & (ids < n_x))[:, None], x[ids.clamp(0, n_x - 1)].double(), 0.0)
        else:
            r = x[b[e]:b[e + 1]].double()
        m = d_y[b[e]:b[e + 1]].double().t().contiguous()
        within(d[e], m @ r, m.abs() @ r.abs(), size, dtype)


def adder(r, m):
    """What the matrix units may lose on E4M3 operands. They add 16 products at a time, all aligned to the largest and
    cut 13 bits below its leading one: at most 16 * 2^-13 of the largest product. (448 * 448 + 2^4 keeps the second
    term, + 2^2 does not; terms of other groups of 16 are added in fp32.)"""
    r, m = (torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 16)).unflatten(1, (-1, 16)).amax(2) for v in (r, m.t()))
    return 2.0 ** -9 * (r @ m.t().contiguous())


def check_fp8(g, sizes, n, k, out_dtype, gather, extra=0):
    rows = sum(sizes) + extra
    gp = offsets(sizes)
    n_x = rows // 3 if gather else rows
    index = torch.randint(0, n_x, (rows,), dtype=torch.int32, device="cuda") if gather else None
    x = rand((n_x, k), torch.bfloat16, 1) * torch.logspace(-2, 2, n_x, device="cuda")[:, None].bfloat16()
    q, s = g.quantise_blocks(x)
    wq, ws = g.quantise_blocks(rand((len(sizes), n, k), torch.float32, 2, k ** -0.5), 128)
    y = g.group_product_fp8(q, s, wq, ws, gp, index=index, out_dtype=out_dtype,
                            out=torch.full((rows, n), float("nan"), dtype=out_dtype, device="cuda"))
    up, down = torch.arange(k, device="cuda") // 128, torch.arange(n, device="cuda") // 128
    xv = q.double() * s.double()[:, up]
    b = gp.tolist()
    for e, size in enumerate(sizes):
        if size:
            r = xv[index[b[e]:b[e + 1]].long()] if gather else xv[b[e]:b[e + 1]]
            m = (wq[e].double() * ws[e].double()[down][:, up]).t().contiguous()
            within(y[b[e]:b[e + 1]], r @ m, r.abs() @ m.abs(), k, out_dtype, adder(r, m))
    assert not y[b[-1]:].any()


@pytest.mark.parametrize("n,k", [(1536, 16), (1536, 128), (1544, 144), (1800, 400), (1536, 1040)])
@pytest.mark.parametrize("gather", [False, True])
def test_large_tiles_fp8(g, n, k, gather):
    check_fp8(g, EDGES, n, k, torch.bfloat16, gather, extra=70 if gather else 0)


@pytest.mark.parametrize("mean", [16, 17, 40, 41, 96, 97, 200])
def test_every_tile_height_fp8(g, mean):
    sizes = [0, 2 * mean, mean // 2, mean + mean - mean // 2, mean - 1, mean + 1]
    for n, k in ((4096 if mean == 16 else 328, 528), (130, 144), (135, 97)):
        check_fp8(g, sizes, n, k, torch.float32, gather=True, extra=3)


def test_large_tiles_do_not_leak(g):
    # NaN and infinities in the padding of rows and matrices, and in rows of other groups
    n, k = 1536, 200
    gp = offsets(EDGES)
    rows = sum(EDGES)
    x, w = rand((rows, k + 8), torch.bfloat16, 1), rand((16, n + 8, k + 8), torch.bfloat16, 2)
    x[:, k:], w[:, n:], w[:, :, k:] = float("nan"), float("inf"), float("nan")
    b = gp.tolist()
    x[b[14]:b[15]] = float("nan")
    y = g.group_product(x[:, :k], w[:, :n, :k], gp)
    assert bool(torch.isnan(y[b[14]:b[15]]).all())
    y[b[14]:b[15]] = 0
    assert bool(torch.isfinite(y).all())
    d = g.group_outer(y, x[:, :k], gp)
    assert bool(torch.isnan(d[14]).all()) and bool(torch.isfinite(d[:14]).all()) and bool(torch.isfinite(d[15:]).all())


@pytest.mark.parametrize("n,k", [(64, 72), (136, 264), (77, 61)])
def test_outer_of_many_long_groups(g, n, k):
    # more than 64 groups, long ones: every 64 are taken in the order of their sizes
    sizes = [260 + 7 * (i % 11) for i in range(64)] + [0, 900, 1, 300, 300]
    rows = sum(sizes)
    gp = offsets(sizes)
    x, d_y = rand((rows, k), torch.bfloat16, 1), rand((rows, n), torch.bfloat16, 2)
    d = g.group_outer(d_y, x, gp, out_dtype=torch.float32)
    b = gp.tolist()
    for e, size in enumerate(sizes):
        m, r = d_y[b[e]:b[e + 1]].double().t().contiguous(), x[b[e]:b[e + 1]].double()
        within(d[e], m @ r, m.abs() @ r.abs(), size, torch.float32)


@pytest.mark.parametrize("rows", [[1, 2], [30, 500], [1500, 900]])
@pytest.mark.parametrize("n,k", [(136, 72), (1536, 128), (61, 45)])
def test_index_into_no_rows(g, rows, n, k):
    # X without a row: whatever the index holds, every result is zero
    total, gp = sum(rows), offsets(rows)
    index = torch.randint(-2, 3, (total,), dtype=torch.int32, device="cuda")
    for pad in (0, 8):
        x = torch.empty((0, k + pad), dtype=torch.bfloat16, device="cuda")[:, :k]
        y = g.group_product(x, rand((2, n, k), torch.bfloat16, 1), gp, index=index)
        assert y.shape == (total, n) and not y.any()
        assert not g.group_product(x, rand((2, k, n), torch.bfloat16, 2), gp, index=index, transposed=True).any()
        assert not g.group_outer(rand((total, n), torch.bfloat16, 3), x, gp, index=index).any()
        q = torch.empty((0, k + 16 * pad), dtype=torch.float8_e4m3fn, device="cuda")[:, :k]
        wq, ws = g.quantise_blocks(rand((2, n, k), torch.float32, 4), 128)
        s = torch.empty((0, -(-k // 128) + pad), device="cuda")[:, :-(-k // 128)]
        assert not g.group_product_fp8(q, s, wq, ws, gp, index=index).any()
