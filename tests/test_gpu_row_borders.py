"""8-bit results at the borders of their roundings: they are those of the division by the scale, value for value."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# ties of E4M3 (halfway between neighbours, the subnormal ones among them) and where values become 0
E4M3_BORDERS = torch.tensor([(j + 0.5) * 2.0 ** -9 for j in range(8)] + [(8 + j + 0.5) / 8 * 2.0 ** e for e in range(-6, 8) for j in range(8)] +
                            [(8 + j + 0.5) * 32 for j in range(6)])


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def near_borders(rows, n, borders, top, exponent, seed, block=128):
    """Rows whose blocks begin with their largest value, `top` times a random scale in 2^exponent .. 2^(exponent + 1), and
    hold borders of the rounding times that scale, or the next value below or above."""
    gen = torch.Generator().manual_seed(seed)
    blocks = -(-n // block)
    scale = (1 + torch.rand((rows, blocks), generator=gen)) * 2.0 ** exponent
    most = scale * top
    scale = most / top
    v = borders[torch.randint(len(borders), (rows, blocks, block), generator=gen)] * scale[..., None]
    which = torch.rand(v.shape, generator=gen)
    up, down = (torch.nextafter(v, torch.full_like(v, to)) for to in (float("inf"), 0.0))
    v = torch.where(which < 1 / 3, up, torch.where(which < 2 / 3, down, v))
    v *= torch.randint(2, v.shape, generator=gen) * 2 - 1
    v[..., 5], v[..., 6] = 0.0, -0.0
    v[..., 0] = most
    return v.flatten(1)[:, :n].contiguous()


def test_borders_are_borders():
    # on the host: rounding the next values up and down of a border in E4M3 and in integers gives neighbours
    t = E4M3_BORDERS
    up, down = torch.nextafter(t, 2 * t), torch.nextafter(t, 0 * t)
    assert bool((up.to(torch.float8_e4m3fn).float() > down.to(torch.float8_e4m3fn).float()).all())


@pytest.mark.parametrize("n", [128, 777, 2056, 20001])
@pytest.mark.parametrize("exponent", [-125, -110, -92, -89, -20, 0, 100])
def test_e4m3_as_quantise_blocks(g, n, exponent):
    """silu(32) is 32 to a unit of 2^-46, so the gate's result is 32 u, exactly; the norm's is whatever its fp32 result is.
    Both are given in fp32 as well, and quantise_blocks of that gives the same bytes."""
    v = near_borders(64 if n < 20000 else 8, n, E4M3_BORDERS, 448.0, exponent, n + exponent)
    h = torch.cat((torch.full_like(v, 32.0), v / 32), 1).cuda()
    r = g.gate(h, quantise=torch.float8_e4m3fn, plain=True)
    q, s = g.quantise_blocks(r.y)
    assert torch.equal(r.scale, s) and torch.equal(r.q.view(torch.uint8), q.view(torch.uint8))
    if exponent > -100:
        assert torch.equal(r.y.cpu(), v)
    # (one row, whose values have a mean square near 1: its results times the weight lie where they happen to)
    x = torch.randn((64, n), generator=torch.Generator().manual_seed(n)).cuda()
    r = g.rms_norm(x, v[0].cuda(), quantise=torch.float8_e4m3fn, plain=True)
    q, s = g.quantise_blocks(r.y)
    assert torch.equal(r.scale, s) and torch.equal(r.q.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("n", [128, 777, 2056, 20001])
@pytest.mark.parametrize("exponent", [-126, -125, -110, -92, -89, 0, 100])
def test_integers_are_the_quotient_rounded(g, n, exponent):
    v = near_borders(64 if n < 20000 else 8, n, torch.arange(127) + 0.5, 127.0, exponent, n + exponent, block=n)
    q, s = g.quantise_rows(v.cuda())
    top = v.abs().amax(1) / 127.0
    assert torch.equal(s.cpu(), top) and bool((top >= 2.0 ** -126).all())
    # (ties, and quotients that are nearer to one than fp32 tells, go to even, as the division's do)
    assert torch.equal(q.cpu().float(), torch.round(v / top[:, None]))
