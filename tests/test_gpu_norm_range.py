"""The norm at the ends of its sums' range: rows whose squares' sum is just below fp32's largest number are right, rows
just above are zeros, and the length of the row is what counts, not its largest value."""
import math

import pytest

from tests import rows_ref as rr
from tests.test_gpu_rows import near

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


@pytest.mark.parametrize("n", [1, 16, 4096, 16384, 20001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ends(g, n, dtype):
    top = math.sqrt(torch.finfo(torch.float32).max)
    x = torch.zeros((4, n))
    x[0] = 0.98 * top / math.sqrt(n)                      # all alike, the squares' sum at 0.96 of the largest number
    x[1, n // 2] = 0.98 * top                             # one alone
    x[2] = 1.02 * top / math.sqrt(n)                      # above
    x[3] = 1e-15                                          # squares of 1e-30
    x = x.to(dtype)
    want = rr.rms_norm(x, None, 1e-30)
    got = g.rms_norm(x.cuda(), None, eps=1e-30).y
    keep = [0, 1, 3]
    # (eps and the smallest row's squares are rounded to fp32, which counts half)
    assert near(got[keep], want[keep], rr.rms_norm_error(want[keep], n) + rr.U32 * want[keep].abs(), dtype)
    assert not got[2].any()
    d = torch.ones_like(x)
    w = torch.ones(n)
    want, mag, _, _ = rr.rms_norm_backward(x[:2], w, d[:2], None, 1e-30)
    d_x, d_w = g.rms_norm_backward(x[:2].cuda(), w.cuda(), d[:2].cuda(), eps=1e-30)
    assert near(d_x, want, rr.backward_error(mag, n), dtype) and bool(torch.isfinite(d_w).all())
