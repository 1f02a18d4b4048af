"""Calls of the routed expert products at the edges of what they accept, against
64-bit forms: infinities and NaN that reach a sum, parts of a routing, scales
near the ends of fp32."""
import dataclasses

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


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("mean", [3, 30, 100, 300])
@pytest.mark.parametrize("experts", [8, 62, 63, 64, 130])
def test_some_of_a_routings_experts(g, transposed, mean, experts):
    # a part of group_ptr with its experts' weights: the other experts' rows are zeros, before and behind
    r = g.route(rand((mean * experts // 2, experts + 7), torch.float32, 1), 2)
    rows = r.token.numel()
    for n, k in ((136, 72), (45, 67)) if experts > 8 else ((136, 72), (45, 67), (2048, 128)):
        x = rand((r.n_tokens, k), torch.bfloat16, 2)
        w = rand((experts,) + ((k, n) if transposed else (n, k)), torch.bfloat16, 3, k ** -0.5)
        gp = r.group_ptr[4:4 + experts + 1]
        y = g.group_product(x, w, gp, index=r.token, transposed=transposed,
                            out=torch.full((rows, n), float("nan"), dtype=torch.bfloat16, device="cuda"))
        b, f = int(gp[0]), int(gp[-1])
        assert 0 < b < f < rows and not y[:b].any() and not y[f:].any()
        whole = g.group_product(x, w, gp - b, index=r.token[b:f].contiguous(), transposed=transposed)
        # (sums in another order where another tile is taken)
        limit = 2.0 ** -7 * whole.double().abs() + (k + 8) * 2.0 ** -22 * float(x.abs().max()) * float(w.abs().max()) * k
        assert bool(((y[b:f].double() - whole.double()).abs() <= limit).all())
        if not transposed:
            q, s = g.quantise_blocks(x)
            wq, ws = g.quantise_blocks(w, 128)
            y = g.group_product_fp8(q, s, wq, ws, gp, index=r.token,
                                    out=torch.full((rows, n), float("nan"), dtype=torch.bfloat16, device="cuda"))
            assert not y[:b].any() and not y[f:].any() and y[b:f].isfinite().all()
            assert y[b:f].any(1).all()


def test_route_refuses_a_top_k_beyond_any_memory(g):
    # refused with a status, before arrays of that many entries are asked for
    for top_k in (9, 1 << 20, 1 << 40):
        with pytest.raises(g.GmagnusError) as e:
            g.route(rand((4096, 8), torch.float32, 1), top_k)
        assert e.value.status == 1


@pytest.mark.parametrize("name,change", [("row_ptr", lambda a: a[:-1]), ("row_ptr", lambda a: a.int()), ("expert", lambda a: a[:-1]),
                                         ("expert", lambda a: a.long()), ("weight", lambda a: a[::2]), ("weight", lambda a: a.half()),
                                         ("weight", lambda a: a.cpu())])
def test_route_backward_refuses_a_routings_arrays(g, name, change):
    # the arrays of a routing that a program put together itself are checked like any other array
    l = rand((20, 8), torch.float32, 1)
    r = g.route(l, 2)
    bad = dataclasses.replace(r, **{name: change(getattr(r, name))})
    with pytest.raises(ValueError, match="routing." + name):
        g.route_backward(l, bad, torch.ones(40, device="cuda"))


def fp8(v):
    return v.to(torch.float8_e4m3fn)


# groups, rows of each, columns, reduction: a work group's 16 rows with 16 and with 64 columns, any alignment, 32, 64 and 256 rows
FP8_SHAPES = [(2, 3, 72, 400), (64, 5, 520, 272), (3, 40, 130, 333), (8, 30, 136, 528), (4, 100, 264, 144), (16, 140, 2048, 272)]


@pytest.mark.parametrize("e,rows,n,k", FP8_SHAPES)
@pytest.mark.parametrize("x_exp,w_exp", [(-63, -63), (-126, 0), (0, -126), (-100, -20), (63, 64), (100, 27), (8, 119)])
def test_fp8_scales_to_the_ends_of_their_product(g, e, rows, n, k, x_exp, w_exp):
    # a block's two scales multiply to between 2^-126 and 2^128: small values meet the large ones, so that sums stay in fp32
    top = 448.0 if x_exp + w_exp < 0 else 2.0 ** -6
    q = fp8(rand((e * rows, k), torch.float32, 1).clamp(-1, 1) * top)
    wq = fp8(rand((e, n, k), torch.float32, 2).clamp(-1, 1) * top)
    kb, nb = -(-k // 128), -(-n // 128)
    mant = lambda shape, seed: 1 + torch.rand(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * 0.4
    s, ws = mant((e * rows, kb), 3) * 2.0 ** x_exp, mant((e, nb, kb), 4) * 2.0 ** w_exp
    q[1, :128] = 0                      # a block whose sum is zero
    y = g.group_product_fp8(q, s, wq, ws, offsets([rows] * e), out_dtype=torch.float32)
    up, down = torch.arange(k, device="cuda") // 128, torch.arange(n, device="cuda") // 128
    xv = (q.double() * s.double()[:, up]).reshape(e, rows, k)
    wv = (wq.double() * ws.double()[:, down][:, :, up]).transpose(1, 2).contiguous()
    want, mag = xv @ wv, xv.abs() @ wv.abs()
    # 16 products at a time are cut 13 bits below the largest: 16 * 2^-13 of it, at most of the sum of magnitudes
    limit = er.U["float32"] * want.abs() + er.TINY["float32"] + ((k + 8) * 2.0 ** -23 + 2.0 ** -9) * mag
    assert y.isfinite().all()
    assert bool(((y.double().reshape(want.shape) - want).abs() <= limit).all())


def test_no_grouped_rows(g):
    # an empty index into an X with rows (no token chose any of these experts): empty results, zero gradients
    x, w = rand((9, 64), torch.bfloat16, 1), rand((3, 72, 64), torch.bfloat16, 2)
    gp, none = offsets([0, 0, 0]), torch.empty(0, dtype=torch.int32, device="cuda")
    assert g.group_product(x, w, gp, index=none).shape == (0, 72)
    assert g.group_product(rand((9, 72), torch.bfloat16, 1), w, gp, index=none, transposed=True).shape == (0, 64)
    d = g.group_outer(torch.empty((0, 72), dtype=torch.bfloat16, device="cuda"), x, gp, index=none,
                      out=torch.full((3, 72, 64), float("nan"), dtype=torch.bfloat16, device="cuda"))
    assert not d.any()
    q, s = g.quantise_blocks(x)
    wq, ws = g.quantise_blocks(w, 128)
    assert g.group_product_fp8(q, s, wq, ws, gp, index=none).shape == (0, 72)
    # and their sums
    y = g.combine(torch.empty((0, 72), dtype=torch.bfloat16, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda"), none)
    assert y.shape == (5, 72) and not y.any()
    d_y, d_w = g.combine_backward(torch.empty((0, 72), dtype=torch.bfloat16, device="cuda"),
                                  torch.zeros(6, dtype=torch.int64, device="cuda"), none, None, y)
    assert d_y.shape == (0, 72) and d_w.shape == (0,)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("normalise", [True, False])
def test_route_weights_of_widely_spread_logits(g, dtype, normalise):
    # logits whose differences are exact in fp32 (multiples of 1/8): the weights are good to a few units however small they are
    t, e = 500, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    l = (torch.randint(0, 84 * 8, (t, e), device="cuda", generator=gen).float() / 8 - 40).to(dtype)
    l[0] = torch.tensor([torch.finfo(dtype).min, 3.0, -float("inf"), 3.0])
    r = g.route(l, e, normalise=normalise)
    want = torch.softmax(l.double(), 1)
    got = torch.zeros(t, e, dtype=torch.float64, device="cuda")
    row = torch.repeat_interleave(torch.arange(t, device="cuda"), r.row_ptr[1:] - r.row_ptr[:-1])
    got[row, r.expert[:row.numel()].long()] = r.weight[:row.numel()].double()
    assert got[0].tolist() == [0.0, 0.5, 0.0, 0.5]
    # units of 2^-24: e^x 5, the sum of 4 terms 4, its reciprocal 3, the product 1
    assert bool(((got - want).abs() <= 13 * 2.0 ** -24 * want + 1e-37).all())
    d = rand((t * e,), torch.float32, 2)
    d64 = torch.zeros_like(got)
    d64[row, r.expert[:row.numel()].long()] = d[:row.numel()].double()
    grad = want * (d64 - (want * d64).sum(1, keepdim=True))
    mag = want * (d64.abs() + (want * d64.abs()).sum(1, keepdim=True))
    limit = er.U[str(dtype).replace("torch.", "")] * grad.abs() + er.TINY[str(dtype).replace("torch.", "")] + 40 * 2.0 ** -24 * mag + 1e-37
    assert bool(((g.route_backward(l, r, d).double() - grad).abs() <= limit).all())


@pytest.mark.parametrize("t,e,k,n", [(50, 12, 3, 40), (400, 70, 2, 520)])
def test_combine_of_some_experts_rows(g, t, e, k, n):
    # the rows of experts 4 .. e - 3 only, slots counted from the first of them: the others add nothing and get no gradient
    r = g.route(rand((t, e), torch.float32, 1), k)
    b, f = int(r.group_ptr[4]), int(r.group_ptr[e - 3])
    y, d_out = rand((t * k, n), torch.bfloat16, 2), rand((t, n), torch.bfloat16, 3)
    here = torch.zeros_like(y)
    here[b:f] = y[b:f]
    slot = r.slot - b
    assert torch.equal(g.combine(y[b:f], r.row_ptr, slot, r.weight), g.combine(here, r.row_ptr, r.slot, r.weight))
    d_y, d_w = g.combine_backward(y[b:f], r.row_ptr, slot, r.weight, d_out)
    want_y, want_w = g.combine_backward(here, r.row_ptr, r.slot, r.weight, d_out)
    assert torch.equal(d_y, want_y[b:f]) and torch.equal(d_w, want_w)
