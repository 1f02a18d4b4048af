"""The layer of a few tokens where a gate's results are small: in fp16 they are kept to 2^-36, not to a subnormal's step."""
import pytest

from tests import rows_ref as rr
from tests.test_gpu_expert_layer_few import dequantised, rand

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

KEPT = {torch.float16: 2.0 ** -36, torch.bfloat16: 2.0 ** -133}  # half a step of the second value, and more


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


@pytest.mark.parametrize("kind", ["16 bits", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens,d,f,n", [(3, 40, 200, 70), (16, 64, 136, 33), (40, 72, 328, 64)])
@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3])
def test_small_results(g, kind, dtype, tokens, d, f, n, size):
    # one expert, weight 1; results of the gate around size^2 / 4, far below 1, and weights that make up for it
    x = rand((tokens, d), dtype, 1, size)
    w1, w2 = rand((1, 2 * f, d), torch.float32, 2, d ** -0.5), rand((1, n, f), torch.float32, 3, 100.0)
    s1 = s2 = None
    if kind == "e4m3":
        (w1, s1), (w2, s2) = g.quantise_blocks(w1, 128), g.quantise_blocks(w2, 128)
    elif kind == "int8":
        (w1, s1), (w2, s2) = g.quantise_rows(w1), g.quantise_rows(w2)
    else:
        w1, w2 = w1.to(dtype), w2.to(dtype)
    y = g.expert_layer(x, torch.zeros((tokens, 1), device="cuda"), 1, w1, w2, w1_scale=s1, w2_scale=s2, out_dtype=torch.float32)
    m1, m2 = dequantised(w1, s1)[0], dequantised(w2, s2)[0]
    h, dh = x.double() @ m1.t(), (d + 8) * 2.0 ** -23 * (x.double().abs() @ m1.abs().t())
    gg, u = h.chunk(2, 1)
    dg, du = dh.chunk(2, 1)
    s = gg * torch.sigmoid(gg)
    a = s * u
    da = (1.1 * dg + 12 * rr.U32 * s.abs()) * (u.abs() + du) + s.abs() * du
    da = da + rr.half_step(dtype) ** 2 * (a.abs() + da) + KEPT[dtype]
    want = a @ m2.t()
    off = da @ m2.abs().t() + (f + 40) * 2.0 ** -23 * ((a.abs() + da) @ m2.abs().t())
    assert bool(((y.double() - want).abs() <= off + rr.U32 * want.abs()).all())
