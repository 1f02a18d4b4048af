"""The norm, the gate and the rounding of rows to 8 bits on the GPU against their 64-bit forms (rows_ref.py)."""
import pytest

from tests import rows_ref as rr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = [torch.float32, torch.bfloat16, torch.float16]
FORMATS = [None, torch.float8_e4m3fn, torch.int8]
# a lane's pieces, the waves of a row and what passes registers: both sides of each border, rows that end inside a piece
COLUMNS = [1, 7, 8, 127, 128, 129, 512, 520, 777, 1024, 1025, 2048, 2056, 3999, 4096, 4104, 8192, 8195, 16384, 16392, 20001]
EPS = 1e-5


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def rand(shape, dtype, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()


def near(got, want, error, dtype):
    want = want.cpu()
    off = (got.double().cpu() - want).abs()
    return bool((off <= rr.half_step(dtype) * (want.abs() + error.cpu()) + error.cpu() + rr.TINY[dtype]).all())


def check_results(r, want, error, dtype, quantise, plain):
    want, error = want.cpu(), error.cpu()
    assert (r.y is not None) == plain and (r.q is not None) == (quantise is not None)
    if plain:
        assert r.y.dtype == dtype and near(r.y, want, error, dtype)
    if quantise is torch.int8:
        rr.check_int8(r.q.cpu(), r.scale.cpu(), want, error)
    elif quantise is not None:
        rr.check_e4m3(r.q.cpu(), r.scale.cpu(), want, error)


def check_norm(g, x, w, res, quantise, plain):
    r = g.rms_norm(x, w, residual=res, eps=EPS, quantise=quantise, plain=plain)
    total = x
    if res is not None:
        total = r.total
        exact = x.double() + res.double()
        # (the sum is rounded to fp32 first, which moves it by no more than that)
        assert near(total, exact, rr.U32 * exact.abs(), x.dtype)
    else:
        assert r.total is None
    want = rr.rms_norm(total.cpu(), None if w is None else w.cpu(), EPS)
    check_results(r, want, rr.rms_norm_error(want, x.shape[1]), x.dtype, quantise, plain or quantise is None)
    return r


@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rms_norm(g, n, dtype):
    rows = 5 if n > 4096 else 19
    x, res = rand((rows, n), dtype, n), rand((rows, n), dtype, n + 1, 3.0)
    w = rand((n,), dtype, n + 2)
    for quantise in FORMATS:
        check_norm(g, x, w, res, quantise, True)
    check_norm(g, x, w.float(), None, torch.float8_e4m3fn, False)
    check_norm(g, x, None, None, None, None)


@pytest.mark.parametrize("rows,n", [(1, 4096), (4, 200), (3000, 264), (8200, 40), (2100, 1032), (1, 1)])
def test_rms_norm_rows(g, rows, n):
    x, res, w = (rand(s, torch.bfloat16, rows + i) for i, s in enumerate([(rows, n), (rows, n), (n,)]))
    for quantise in FORMATS:
        check_norm(g, x, w, res, quantise, True)


@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rms_norm_backward(g, n, dtype):
    rows = 5 if n > 4096 else 37
    h, d, dt = (rand((rows, n), dtype, n + i) for i in range(3))
    for w in (rand((n,), dtype, n + 5), rand((n,), torch.float32, n + 6), None):
        for d_total in (dt, None):
            d_x, d_w = g.rms_norm_backward(h, w, d, d_total=d_total, eps=EPS)
            want, mag, want_w, mag_w = rr.rms_norm_backward(*(None if t is None else t.cpu() for t in (h, w, d, d_total)), EPS)
            assert d_x.dtype == dtype and near(d_x, want, rr.backward_error(mag, n), dtype)
            if w is None:
                assert d_w is None
            else:
                assert d_w.dtype == torch.float32 and near(d_w, want_w, rr.weight_error(mag_w, rows, n), torch.float32)


@pytest.mark.parametrize("rows,n", [(1, 4096), (3, 64), (2500, 264), (9000, 48), (700, 2056), (600, 16400), (1, 1)])
def test_rms_norm_backward_rows(g, rows, n):
    h, d = rand((rows, n), torch.bfloat16, rows), rand((rows, n), torch.bfloat16, rows + 1)
    w = rand((n,), torch.bfloat16, 3)
    d_x, d_w = g.rms_norm_backward(h, w, d, eps=EPS)
    want, mag, want_w, mag_w = rr.rms_norm_backward(h.cpu(), w.cpu(), d.cpu(), None, EPS)
    assert near(d_x, want, rr.backward_error(mag, n), torch.bfloat16)
    assert near(d_w, want_w, rr.weight_error(mag_w, rows, n), torch.float32)
    again = g.rms_norm_backward(h, w, d, eps=EPS)
    assert torch.equal(d_x, again[0]) and torch.equal(d_w, again[1])


def test_rms_norm_gradients_against_differences(g):
    x, w, d, dt = rand((4, 50), torch.float32, 1), rand((50,), torch.float32, 2), rand((4, 50), torch.float32, 3), rand((4, 50), torch.float32, 4)
    d_x, d_w = (t.double().cpu() for t in g.rms_norm_backward(x, w, d, d_total=dt, eps=EPS))
    x, w, d, dt = (t.double().cpu() for t in (x, w, d, dt))

    def loss(x, w):
        return float((rr.rms_norm(x, w, EPS) * d).sum() + (x * dt).sum())

    for seed in range(6):
        gen = torch.Generator().manual_seed(seed)
        vx, vw = torch.randn(4, 50, generator=gen, dtype=torch.float64), torch.randn(50, generator=gen, dtype=torch.float64)
        step = 1e-5
        slope = (loss(x + step * vx, w + step * vw) - loss(x - step * vx, w - step * vw)) / (2 * step)
        # third derivatives times step^2, cancellation 1e-16 / step, and fp32 gradients of some 250 terms
        assert abs(slope - float((d_x * vx).sum() + (d_w * vw).sum())) <= 1e-4


@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("dtype", TYPES)
def test_gate(g, n, dtype):
    rows = 5 if n > 4096 else 19
    h = rand((rows, 2 * n), dtype, n, 3.0)
    want = rr.gate(h.cpu())
    for quantise in FORMATS:
        for plain in (True, False):
            check_results(g.gate(h, quantise=quantise, plain=plain or quantise is None), want, rr.gate_error(want, h.cpu()), dtype,
                          quantise, plain or quantise is None)
    d = rand((rows, n), dtype, n + 1)
    got = g.gate_backward(h, d)
    want, mag = rr.gate_backward(h.cpu(), d.cpu())
    assert got.dtype == dtype and near(got, want, rr.gate_backward_error(mag, h.cpu(), d.cpu()), dtype)


def test_gate_far_values(g):
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1.0, -1.0, -1.2784645, 20.0, -20.0, 87.0, -87.0, -88.5, -95.0, -150.0, -1e4, 1e4, 3e38, -3e38])
    h = torch.stack((v, torch.full_like(v, 0.5)), 1).cuda()
    want = rr.gate(h.cpu())
    assert near(g.gate(h).y, want, rr.gate_error(want, h.cpu()), torch.float32)
    got = g.gate_backward(h, torch.ones_like(h[:, :1]))
    want, mag = rr.gate_backward(h.cpu(), torch.ones(len(v), 1))
    assert near(got, want, rr.gate_backward_error(mag, h.cpu(), torch.ones(len(v), 1)), torch.float32)


def test_gate_gradient_against_differences(g):
    h, d = rand((3, 40), torch.float32, 1), rand((3, 20), torch.float32, 2)
    got = g.gate_backward(h, d).double().cpu()
    h, d = h.double().cpu(), d.double().cpu()
    for seed in range(5):
        v = torch.randn(3, 40, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
        slope = float(((rr.gate(h + 1e-5 * v) - rr.gate(h - 1e-5 * v)) * d).sum()) / 2e-5
        assert abs(slope - float((got * v).sum())) <= 1e-4


@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_rows(g, n, dtype):
    x = rand((7, n), dtype, n, 5.0)
    x[2] = 0
    x[3] *= 1e-3
    q, s = g.quantise_rows(x)
    want = x.double().cpu()
    rr.check_int8(q.cpu(), s.cpu(), want, torch.zeros_like(want))
    assert not q[2].any() and float(s[2]) == 2.0 ** -126


def test_quantise_rows_of_a_stack(g):
    x = rand((5, 33, 200), torch.bfloat16, 1)[:, 3:, 8:]
    q, s = g.quantise_rows(x)
    assert q.shape == (5, 30, 192) and s.shape == (5, 30)
    for i in range(5):
        one, s1 = g.quantise_rows(x[i])
        assert torch.equal(q[i], one) and torch.equal(s[i], s1)


def test_ties_go_to_even(g):
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]]).cuda()
    q, s = g.quantise_rows(x)
    assert float(s[0]) == 1.0 and q[0].tolist() == [127, 0, 2, 2, 0, -2, -2, 126]


@pytest.mark.parametrize("n", [8, 300, 4097, 20001])
def test_integers_at_the_ends_of_fp32(g, n):
    x = rand((6, n), torch.float32, n)
    x /= x.abs().amax(1, keepdim=True)
    top = torch.tensor([torch.finfo(torch.float32).max, 2.0 ** -118, 2.0 ** -120, 2.0 ** -126, 2.0 ** -130, 2.0 ** -149], device="cuda")
    x *= top[:, None]
    q, s = g.quantise_rows(x)
    want = x.double().cpu()
    rr.check_int8(q.cpu(), s.cpu(), want, torch.zeros_like(want))
    assert bool((s[2:] == 2.0 ** -126).all())


@pytest.mark.parametrize("n", [8, 300, 4097, 20001])
@pytest.mark.parametrize("top", [3e37, 1e-35, 1e-38, 1e-41])
def test_8_bit_results_at_the_ends_of_fp32(g, n, top):
    """Values stay below 10 times the weight. Among subnormals a rounding takes 2^-150, here two: 2^-149, and 2^-148 counted."""
    x = rand((5, n), torch.float32, n)
    w = torch.full((n,), top, device="cuda")
    want = rr.rms_norm(x.cpu(), w.cpu(), EPS)
    assert float(want.abs().max()) < 10 * top
    error = rr.rms_norm_error(want, n) + 2.0 ** -148
    for quantise in (torch.int8, torch.float8_e4m3fn):
        check_results(g.rms_norm(x, w, eps=EPS, quantise=quantise, plain=True), want, error, torch.float32, quantise, True)


@pytest.mark.parametrize("off", [1, 3, 8])
@pytest.mark.parametrize("n", [200, 777, 4099])
def test_strided_and_unaligned_rows(g, n, off):
    wide, res, d = (rand((9, 2 * n + 24), torch.float16, i) for i in range(3))
    w = rand((n + 8,), torch.float16, 4)
    x, r, dy, h = wide[:, off:off + n], res[:, off + 1:off + 1 + n], d[:, off + 2:off + 2 + n], wide[:, off:off + 2 * n]
    for quantise in FORMATS:
        a = g.rms_norm(x, w[off:off + n], residual=r, quantise=quantise, plain=True)
        b = g.rms_norm(x.contiguous(), w[off:off + n].contiguous(), residual=r.contiguous(), quantise=quantise, plain=True)
        c, e = g.gate(h, quantise=quantise, plain=True), g.gate(h.contiguous(), quantise=quantise, plain=True)
        for p, q in zip(tuple(a) + tuple(c), tuple(b) + tuple(e)):
            assert (p is None and q is None) or torch.equal(p.view(torch.uint8), q.view(torch.uint8))
    a, b = g.rms_norm_backward(x, w[off:off + n], dy), g.rms_norm_backward(x.contiguous(), w[off:off + n].contiguous(), dy.contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    buf = torch.full((9, 2 * n + 32), 7.0, dtype=torch.float16, device="cuda")
    out = g.gate_backward(h, dy, out=buf[:, 5:5 + 2 * n])
    assert torch.equal(out, g.gate_backward(h.contiguous(), dy.contiguous()))
    assert bool((buf[:, :5] == 7).all()) and bool((buf[:, 5 + 2 * n:] == 7).all())


def test_infinities_and_nans_stay_in_their_rows(g):
    for n in (136, 4096, 20000):
        x = rand((6, n), torch.float32, n)
        clean = g.rms_norm(x, None, quantise=torch.int8, plain=True)
        bad = x.clone()
        bad[1, 5], bad[3, n - 1] = float("nan"), float("inf")
        for quantise in (torch.int8, torch.float8_e4m3fn):
            r = g.rms_norm(bad, None, quantise=quantise, plain=True)
            assert bool(torch.isnan(r.y[1]).all()) and bool(torch.isnan(r.y[3, n - 1]))
            assert bool(torch.isnan(r.scale[1]).all())
            for i in (0, 2, 4, 5):
                assert torch.equal(r.y[i], clean.y[i])
        q, s = g.quantise_rows(bad)
        values = q.float() * s[:, None]
        assert bool(torch.isnan(s[1])) and bool(torch.isnan(values[1]).all()) and bool(torch.isinf(s[3])) and bool(torch.isnan(values[3]).all())
        assert torch.equal(q[0], g.quantise_rows(x)[0][0])


def test_zero_rows_and_no_rows(g):
    z = torch.zeros((3, 300), dtype=torch.bfloat16, device="cuda")
    r = g.rms_norm(z, None, residual=z, quantise=torch.float8_e4m3fn, plain=True)
    assert not r.y.any() and not r.q.float().any() and bool((r.scale == 2.0 ** -126).all())
    d_x, d_w = g.rms_norm_backward(z, torch.ones(300, device="cuda"), z + 1)
    assert bool(torch.isfinite(d_x).all()) and not d_w.any()
    none = z[:0]
    r = g.rms_norm(none, None, residual=none, quantise=torch.int8, plain=True)
    assert r.y.shape == (0, 300) and r.scale.shape == (0,)
    d_x, d_w = g.rms_norm_backward(none, torch.ones(300, device="cuda"), none)
    assert d_x.shape == (0, 300) and not d_w.any() and d_w.shape == (300,)
    assert g.gate(none).y.shape == (0, 150) and g.gate_backward(none, none[:, :150]).shape == (0, 300)
    assert g.quantise_rows(none)[0].shape == (0, 300) and g.quantise_rows(z[None][:0])[1].shape == (0, 3)


def test_other_stream_and_graph(g):
    x, res, w, d = rand((300, 1000), torch.bfloat16, 1), rand((300, 1000), torch.bfloat16, 2), rand((1000,), torch.bfloat16, 3), rand((300, 1000), torch.bfloat16, 4)

    def work():
        r = g.rms_norm(x, w, residual=res, quantise=torch.float8_e4m3fn, plain=True)
        b = g.rms_norm_backward(r.total, w, d, d_total=d)
        c = g.gate(r.y, quantise=torch.int8, plain=True)
        return [r.y, r.q.view(torch.uint8), r.scale, r.total, b[0], b[1], c.y, c.q, c.scale, g.gate_backward(r.y, c.y)]

    want = [t.clone() for t in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = g.rms_norm(x, w, residual=res, stream=side)
    b = g.rms_norm_backward(r.total, w, d, d_total=d, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(r.y, want[0]) and torch.equal(b[0], want[4]) and torch.equal(b[1], want[5])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for turn in range(4):
        x.copy_(rand((300, 1000), torch.bfloat16, 10 + turn))
        want = [t.clone() for t in work()]
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_rows_past_32_bit_offsets(g):
    # 2^31 elements and more before the last rows
    wide = torch.zeros((3, (1 << 30) + 64), dtype=torch.bfloat16, device="cuda")
    x, h = wide[:, :1000], wide[:, :2000]
    x.copy_(rand((3, 1000), torch.bfloat16, 1))
    r, want = g.rms_norm(x, None, quantise=torch.int8, plain=True), g.rms_norm(x.contiguous(), None, quantise=torch.int8, plain=True)
    assert torch.equal(r.y, want.y) and torch.equal(r.q, want.q)
    assert torch.equal(g.gate(h).y, g.gate(h.contiguous()).y)


def test_differentiating_raises(g):
    x, w = rand((4, 64), torch.bfloat16, 1), rand((64,), torch.bfloat16, 2)
    for name, call in (("rms_norm", lambda t: g.rms_norm(t, w, residual=x)), ("rms_norm", lambda t: g.rms_norm(x, w, residual=t)),
                       ("rms_norm", lambda t: g.rms_norm(x, t[0], quantise=torch.int8)), ("gate", lambda t: g.gate(t)),
                       ("quantise_rows", lambda t: g.Rows(None, *g.quantise_rows(t), None))):
        r = call(x.clone().requires_grad_())
        for t in r:
            if t is not None and t.dtype != torch.int8:
                with pytest.raises(RuntimeError, match="gmagnus.%s has no autograd formula" % name):
                    t.float().sum().backward()


def test_binding_refuses(g):
    x, w = rand((4, 64), torch.bfloat16, 1), rand((64,), torch.bfloat16, 2)
    for call in (lambda: g.rms_norm(x, w[:63]), lambda: g.rms_norm(x, w.half()), lambda: g.rms_norm(x, w, quantise=torch.uint8),
                 lambda: g.rms_norm(x[0], w), lambda: g.gate(x[:, :63]), lambda: g.rms_norm(x.to(torch.int8), None),
                 lambda: g.rms_norm_backward(x, w[::2], x), lambda: g.quantise_rows(x.int()), lambda: g.rms_norm(x.t(), None),
                 lambda: g.gate_backward(x, x[:, :32], out=x[:, :32])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: g.rms_norm(x, w, residual=x[:3]), lambda: g.rms_norm(x, w, residual=x.half()), lambda: g.rms_norm(x, w, plain=False),
                 lambda: g.rms_norm(x, w, eps=-1.0), lambda: g.rms_norm(x, w, eps=float("nan")), lambda: g.rms_norm_backward(x, w, x[:, :63]),
                 lambda: g.gate_backward(x, x), lambda: g.gate(x, plain=False)):
        with pytest.raises(g.GmagnusError) as e:
            call()
        assert e.value.status == 1
