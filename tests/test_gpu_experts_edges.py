"""Calls of the routed expert products at the edges of what they accept, against
64-bit forms: infinities and NaN that reach a sum, parts of a routing, scales
near the ends of fp32."""
import numpy as np
import pytest

from tests import experts_ref as er

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("e", [9, 70, 300])
def test_route_backward_masked_logits_get_zero(g, bad, normalise, e):
    # a NaN or an infinity among a row's gradients or logits reaches neither masked logits nor other rows
    t, k = 12, 3
    l = rand((t, e), torch.float32, e)
    l[:, 4:6] = -float("inf")
    l[:, 7] = float("nan")
    r = g.route(l, k, normalise=normalise)
    d = rand((t * k,), torch.float32, 1)
    d[1 * k + 2] = bad                  # row 1's last entry
    clean = g.route_backward(l, r, torch.where(d.isfinite(), d, 0.0))
    out = g.route_backward(l, r, d)
    rows = [i for i in range(t) if i != 1]
    assert torch.equal(out[rows], clean[rows])
    assert not out[:, 4:6].any() and not out[:, 7].any()
    chosen = torch.zeros(e, dtype=torch.bool, device="cuda")
    chosen[r.expert[k:2 * k].long()] = True
    assert not out[1, chosen].isfinite().any()
    if normalise:                       # the weights do not depend on what was not chosen
        assert not out[1, ~chosen].any()
    l[2, 3] = float("inf")              # a NaN weight, in the sum of its own row
    r = g.route(l, k, normalise=normalise)
    out = g.route_backward(l, r, torch.ones(t * k, device="cuda"))
    assert not out[:, 4:6].any() and not out[:, 7].any() and out[rows[2:]].isfinite().all()
