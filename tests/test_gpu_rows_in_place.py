"""Outputs that are an input itself: the same results as with memory of their own, however long the rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

COLUMNS = [300, 777, 4096, 8200, 16384, 16392, 20001]


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


def rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def stream():
    return torch.cuda.current_stream().cuda_stream


def norm(g, x, residual, w, total, y, q, scale):
    d = [None if t is None else g._dense(t, 0, "t", int8=True) for t in (x, residual, w[None], total, y, q, scale)]
    g._check(g.load().gmagnus_rms_norm(d[0], d[1], d[2], 1e-5, *d[3:], stream()))


@pytest.mark.parametrize("n", COLUMNS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("quantise", [None, torch.int8, torch.float8_e4m3fn])
def test_norm(g, n, dtype, quantise):
    rows = 9 if n > 4096 else 40
    x, res, w = rand((rows, n), dtype, 1), rand((rows, n), dtype, 2), rand((n,), dtype, 3)
    want = g.rms_norm(x, w, residual=res, eps=1e-5, quantise=quantise, plain=True)
    alone = g.rms_norm(x, w, eps=1e-5, quantise=quantise, plain=True)
    for total_is, y_is in (("residual", None), ("x", None), ("residual", "x"), ("x", "residual"), (None, "x"), (None, "residual"), ("none", "x")):
        a = dict(x=x.clone(), residual=res.clone())
        total = None if total_is == "none" else a.get(total_is, torch.empty_like(x))
        y = a.get(y_is, torch.empty_like(x))
        q = None if quantise is None else torch.empty((rows, n), dtype=quantise, device="cuda")
        scale = None if q is None else torch.empty((1, rows) if quantise is torch.int8 else (rows, -(-n // 128)), device="cuda")
        norm(g, a["x"], None if total is None else a["residual"], w, total, y, q, scale)
        r = alone if total is None else want
        assert torch.equal(y, r.y) and (total is None or torch.equal(total, r.total)), (total_is, y_is)
        if q is not None:
            assert torch.equal(q.view(torch.uint8), r.q.view(torch.uint8)) and torch.equal(scale.flatten(), r.scale.flatten())


@pytest.mark.parametrize("n", COLUMNS)
def test_gradients(g, n):
    rows = 9 if n > 4096 else 40
    h, d, t = (rand((rows, n), torch.bfloat16, i) for i in range(3))
    w = rand((n,), torch.bfloat16, 4)
    want_x, want_w = g.rms_norm_backward(h, w, d, d_total=t, eps=1e-5)
    lib = g.load()
    nbytes = lib.gmagnus_rms_norm_backward_workspace_bytes(rows, n)
    for place in range(3):
        m = [v.clone() for v in (h, d, t)]
        ws, d_w = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda")
        ds = [g._dense(v, 0, "v") for v in m]
        g._check(lib.gmagnus_rms_norm_backward(ds[0], g._dense(w[None], 0, "w"), 1e-5, ds[1], ds[2], ds[place], d_w.data_ptr(), ws.data_ptr(),
                                               nbytes, stream()))
        assert torch.equal(m[place], want_x) and torch.equal(d_w, want_w)
    pair, d_a = rand((rows, 2 * n), torch.float16, 5), rand((rows, n), torch.float16, 6)
    pair[0, :n] = -100.0  # (read again there)
    want = g.gate_backward(pair, d_a)
    assert torch.equal(g.gate_backward(pair, d_a, out=pair), want) and torch.equal(pair, want)
