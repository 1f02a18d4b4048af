"""A whole layer of gated experts for a few tokens in one call, against its 64-bit form.

Errors are followed through: fp32 sums of K products are off by at most 2^-23 K times the sum of magnitudes, silu's
slope is below 1.1, the gate's result is held as two values of the rows' type (half a step of it, squared, is off; below
the normal range half a subnormal's step) and the layer's result is rounded to its type."""
import numpy as np
import pytest

from tests import experts_ref as er
from tests import rows_ref as rr

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
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()


def dequantised(w, scale):
    if scale is None:
        return w.double()
    if w.dtype == torch.int8:
        return w.double() * scale.double()[..., None]
    n, k = w.shape[-2:]
    return w.double() * scale.double().repeat_interleave(128, -2).repeat_interleave(128, -1)[..., :n, :k]


def reference(x, logits, top_k, normalise, w1, w2):
    """(result, how far one in fp32 with a gate's result in x's type may be from it), both float64."""
    r = er.route(logits.double().cpu().numpy(), top_k, normalise)
    t, f = x.shape[0], w2.shape[2]
    out = torch.zeros(t, w2.shape[1], dtype=torch.float64, device="cuda")
    off = torch.zeros_like(out)
    l = logits.double().cpu().numpy()
    far = 2 * np.abs(np.where(np.isfinite(l), l, 0.0)).max(initial=0.0)
    weight_rel = (far + logits.shape[1] + 8) * 2.0 ** -23
    terms = f * top_k
    for e in range(w1.shape[0]):
        b, n = r["group_ptr"][e], r["group_ptr"][e + 1]
        if b == n:
            continue
        ids = torch.from_numpy(r["token"][b:n].astype(np.int64)).cuda()
        wt = torch.from_numpy(r["group_weight"][b:n]).cuda()[:, None]
        xs, m1, m2 = x[ids].double(), w1(e), w2[e] if not callable(w2) else w2(e)
        h, dh = xs @ m1.t(), (x.shape[1] + 8) * 2.0 ** -23 * (xs.abs() @ m1.abs().t())
        gg, u = h.chunk(2, 1)
        dg, du = dh.chunk(2, 1)
        s = gg * torch.sigmoid(gg)
        a = s * u
        da = (1.1 * dg + 12 * rr.U32 * s.abs()) * (u.abs() + du) + s.abs() * du + 2.0 ** -125 * (1 + (gg * u).abs())
        da = da + rr.half_step(x.dtype) ** 2 * (a.abs() + da) + rr.TINY[x.dtype]
        y, mag = a @ m2.t(), (a.abs() + da) @ m2.abs().t()
        out[ids] += wt * y
        off[ids] += wt * (da @ m2.abs().t() + ((terms + 40) * 2.0 ** -23 + weight_rel) * mag)
        # a gate's result beyond its type's range is infinite, and its token's results are infinities and NaN
        off[ids[(a.abs() + da > torch.finfo(x.dtype).max).any(1)]] = float("inf")
    return out, off


class Stack:
    """A stack's matrices in float64, one at a time."""

    def __init__(self, w, scale):
        self.w, self.scale, self.shape = w, scale, w.shape

    def __call__(self, e):
        return dequantised(self.w[e], None if self.scale is None else self.scale[e])


def check(g, x, logits, top_k, w1, w2, normalise=True, s1=None, s2=None, out_dtype=None, **kw):
    n = w2.shape[1]
    y = g.expert_layer(x, logits, top_k, w1, w2, normalise=normalise, w1_scale=s1, w2_scale=s2, out_dtype=out_dtype, **kw)
    want, off = reference(x, logits, top_k, normalise, Stack(w1, s1), Stack(w2, s2))
    dtype = out_dtype or x.dtype
    assert y.dtype == dtype and y.shape == (x.shape[0], n)
    near = (y.double() - want).abs() <= off + rr.half_step(dtype) * (want.abs() + off) + rr.TINY[dtype]
    over = want.abs() + off > torch.finfo(dtype).max
    assert bool((near | over).all())
    return y


def case(t, e, d, f, n, dtype, seed=0, fp8=False):
    x, logits = rand((t, d), dtype, seed + 1), rand((t, e), torch.float32, seed + 2, 1.5)
    w1, w2 = rand((e, 2 * f, d), torch.float32, seed + 3, d ** -0.5), rand((e, n, f), torch.float32, seed + 4, f ** -0.5)
    return x, logits, w1 if fp8 else w1.to(dtype), w2 if fp8 else w2.to(dtype)


# tokens, experts, top_k, hidden, inner, outputs: 16 rows of an expert and more, blocks of 64 and 128 and what is left of
# them, chunks of four blocks and runs of 16, tiles that end inside 16 gates and 32 outputs, one split and several
SIZES = [(1, 1, 1, 1, 1, 1), (1, 4, 2, 64, 16, 32), (1, 16, 2, 256, 128, 256), (2, 8, 8, 63, 17, 33), (5, 64, 4, 1024, 520, 200),
         (15, 3, 2, 130, 250, 96), (16, 64, 6, 192, 256, 64), (17, 2, 2, 129, 257, 31), (33, 5, 1, 320, 72, 100),
         (64, 2, 1, 777, 129, 333), (64, 1, 1, 2056, 1032, 40), (64, 8, 3, 512, 300, 1030), (48, 65, 8, 200, 200, 200),
         (31, 256, 8, 96, 64, 48), (20, 300, 2, 72, 40, 24), (7, 1024, 16, 64, 24, 40), (64, 1024, 16, 32, 16, 8)]


@pytest.mark.parametrize("t,e,k,d,f,n", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_16bit_weights(g, t, e, k, d, f, n, dtype):
    x, logits, w1, w2 = case(t, e, d, f, n, dtype)
    check(g, x, logits, k, w1, w2)
    check(g, x, logits, k, w1, w2, normalise=False, out_dtype=torch.float32)


@pytest.mark.parametrize("t,e,k,d,f,n", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_e4m3_weights(g, t, e, k, d, f, n, dtype):
    x, logits, w1, w2 = case(t, e, d, f, n, dtype, fp8=True)
    (q1, s1), (q2, s2) = g.quantise_blocks(w1, 128), g.quantise_blocks(w2, 128)
    check(g, x, logits, k, q1, q2, s1=s1, s2=s2)
    check(g, x, logits, k, q1, q2, s1=s1, s2=s2, normalise=False, out_dtype=torch.float32)


@pytest.mark.parametrize("t,e,k,d,f,n", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_integer_weights(g, t, e, k, d, f, n, dtype):
    x, logits, w1, w2 = case(t, e, d, f, n, dtype, fp8=True)
    (q1, s1), (q2, s2) = g.quantise_rows(w1), g.quantise_rows(w2)
    check(g, x, logits, k, q1, q2, s1=s1, s2=s2)
    check(g, x, logits, k, q1, q2, s1=s1, s2=s2, normalise=False, out_dtype=torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_integer_and_every_e4m3_value_is_widened_exactly(g, dtype):
    # one expert, a gate of one (silu(g) is g to a unit at g = 24): each result is a weight of W2 times what the gate gives
    x = torch.ones((1, 16), dtype=dtype, device="cuda")
    values = torch.arange(256, dtype=torch.uint8, device="cuda")
    gate = torch.zeros((2 * 256, 16), device="cuda")
    gate[:256, 0], gate[256:, 0] = 24.0, 1.0 / 24.0
    one = torch.zeros((1, 1), device="cuda")
    # W2 has row i with value i at place i
    for kind in (torch.int8, torch.float8_e4m3fn):
        w2 = torch.zeros((1, 256, 256), dtype=torch.uint8, device="cuda")
        w2[0].diagonal().copy_(values)
        w2 = w2.view(kind)
        if kind is torch.int8:
            (q1, s1), s2 = g.quantise_rows(gate[None]), torch.ones((1, 256), device="cuda")
        else:
            (q1, s1), s2 = g.quantise_blocks(gate[None], 128), torch.ones((1, 2, 2), device="cuda")
        want = w2[0].double().diagonal()
        h = dequantised(q1, s1)[0] @ x[0].double()
        unit = (h[:256] * torch.sigmoid(h[:256]) * h[256:])
        y = g.expert_layer(x, one, 1, q1, w2, w1_scale=s1, w2_scale=s2, out_dtype=torch.float32)[0].double()
        nan = torch.isnan(want)  # (a NaN of E4M3 makes its own result NaN)
        assert torch.equal(torch.isnan(y), nan)
        assert bool(((y - want * unit).abs() <= 40 * 2.0 ** -24 * (want * unit).abs() + rr.half_step(dtype) ** 2 * want.abs())[~nan].all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_masked_logits_of_any_type(g, fp8, dtype):
    x, logits, w1, w2 = case(20, 70, 96, 48, 64, torch.bfloat16, fp8=fp8)
    logits[:, 5:9] = -float("inf")
    logits[1] = -float("inf")               # a token without experts
    logits[2, :68] = -float("inf")          # fewer than top_k
    logits[3] = 1.5                         # ties: the lowest experts
    logits[4, 10:20] = float("nan")         # masked
    logits = logits.to(dtype)
    s1 = s2 = None
    if fp8:
        (w1, s1), (w2, s2) = g.quantise_blocks(w1, 128), g.quantise_blocks(w2, 128)
    y = check(g, x, logits, 4, w1, w2, s1=s1, s2=s2)
    assert not y[1].any() and bool(torch.isfinite(y).all())
    none = g.expert_layer(x, torch.full_like(logits, -float("inf")), 4, w1, w2, w1_scale=s1, w2_scale=s2)
    assert not none.any()


@pytest.mark.parametrize("t", [3, 20, 64])
def test_same_choice_as_route(g, t):
    # the layer's parts one after the other: rounded once more in between, so both are near the 64-bit form
    x, logits, w1, w2 = case(t, 16, 256, 128, 256, torch.float16)
    r = g.route(logits, 3)
    a = g.gate(g.group_product(x, w1, r.group_ptr, index=r.token)).y
    y = g.combine(g.group_product(a, w2, r.group_ptr, out_dtype=torch.float32), r.row_ptr, r.slot, r.weight)
    one = check(g, x, logits, 3, w1, w2, out_dtype=torch.float32)
    # the gate's operands and result are rounded to fp16 in between: three half steps on sums of 128 terms at most
    want, off = reference(x, logits, 3, True, Stack(w1, None), Stack(w2, None))
    assert float((y.double() - want).norm() / want.norm()) <= 4 * 2.0 ** -11 and float((one - y).norm() / y.norm()) <= 8 * 2.0 ** -11


def test_weights_of_other_experts_do_not_matter(g):
    x, logits, w1, w2 = case(18, 6, 192, 80, 72, torch.bfloat16)
    logits[:, 4] = -float("inf")
    logits[1:, 2] = -float("inf")
    logits[0, 2] = 9.0                       # expert 2 is token 0's alone
    want = g.expert_layer(x, logits, 2, w1, w2)
    w1[4], w2[4] = float("nan"), float("inf")
    assert torch.equal(g.expert_layer(x, logits, 2, w1, w2), want)
    w1[2], w2[2] = float("nan"), float("inf")
    y = g.expert_layer(x, logits, 2, w1, w2)
    assert bool(torch.isnan(y[0]).all()) and torch.equal(y[1:], want[1:])
    x[5, 7] = float("inf")
    y = g.expert_layer(x, logits, 2, w1, w2)
    assert not bool(torch.isfinite(y[5]).any()) and torch.equal(y[1:5], want[1:5]) and torch.equal(y[6:], want[6:])


def test_infinite_logit_gives_nan_as_route_does(g):
    x, logits, w1, w2 = case(4, 8, 64, 32, 32, torch.bfloat16)
    want = g.expert_layer(x, logits, 2, w1, w2)
    logits[2, 3] = float("inf")
    y = g.expert_layer(x, logits, 2, w1, w2)
    assert bool(torch.isnan(y[2]).all()) and torch.equal(y[[0, 1, 3]], want[[0, 1, 3]])


@pytest.mark.parametrize("scale", [1.0, 0.002])  # (E4M3 values up to 448: the first passes fp16's range)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("off", [1, 8, 16])
def test_strides_and_alignment(g, fp8, off, scale):
    x, logits, w1, w2 = case(19, 6, 300 + off, 130 + off, 90 + off, torch.float16, fp8=fp8)
    s1 = s2 = None
    if fp8:
        (w1, _), (w2, _) = g.quantise_blocks(w1, 128), g.quantise_blocks(w2, 128)
        s1, s2 = (rand((6, 5, 9), torch.float32, 9 + i).abs() * scale for i in range(2))
    x, logits, w1 = x[:, off:], torch.cat((logits, logits), 1)[:, 3:9], w1[:, :2 * 130, off:]
    w2 = w2[:, off:, off:]
    if fp8:
        s1, s2 = s1[:, 1:4, 2:5], s2[:, 2:3, 1:3]
    buf = torch.full((19, 90 + 16), 5.0, dtype=torch.float16, device="cuda")
    a = check(g, x, logits, 2, w1, w2, s1=s1, s2=s2, out=buf[:, 3:93])
    b = g.expert_layer(*(v.contiguous() for v in (x, logits)), 2, *(v.contiguous() for v in (w1, w2)),
                       w1_scale=None if s1 is None else s1.contiguous(), w2_scale=None if s2 is None else s2.contiguous())
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and bool((buf[:, :3] == 5).all()) and bool((buf[:, 93:] == 5).all())


def test_weights_past_32_bit_offsets(g):
    # two experts more than 2^32 bytes apart
    big = torch.zeros((2, (1 << 31) + 4096), dtype=torch.bfloat16, device="cuda")
    x, logits, w1, w2 = case(3, 2, 64, 32, 48, torch.bfloat16)
    v1 = big[:, :2 * 32 * 64].unflatten(1, (64, 64))
    v2 = big[:, 4096:4096 + 48 * 32].unflatten(1, (48, 32))
    v1.copy_(w1)
    v2.copy_(w2)
    assert torch.equal(g.expert_layer(x, logits, 2, v1, v2), g.expert_layer(x, logits, 2, w1, w2))


@pytest.mark.parametrize("fp8", [False, True])
def test_runs_agree_streams_and_graphs(g, fp8):
    x, logits, w1, w2 = case(24, 32, 512, 384, 512, torch.bfloat16, fp8=fp8)
    s1 = s2 = None
    if fp8:
        (w1, s1), (w2, s2) = g.quantise_blocks(w1, 128), g.quantise_blocks(w2, 128)

    def work():
        return g.expert_layer(x, logits, 4, w1, w2, w1_scale=s1, w2_scale=s2)

    want = work()
    for _ in range(20):
        assert torch.equal(work(), want)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for turn in range(12):  # several at once
        s = streams[turn % 3]
        s.wait_stream(torch.cuda.current_stream())
        got.append(g.expert_layer(x, logits, 4, w1, w2, w1_scale=s1, w2_scale=s2, stream=s))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(y, want) for y in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for turn in range(4):
        x.copy_(rand((24, 512), torch.bfloat16, 30 + turn))
        logits.copy_(rand((24, 32), torch.float32, 40 + turn))
        want = work()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_tokens_and_refusals(g):
    x, logits, w1, w2 = case(4, 8, 64, 32, 48, torch.bfloat16)
    assert g.expert_layer(x[:0], logits[:0], 2, w1, w2).shape == (0, 48)
    for call in (lambda: g.expert_layer(x, logits, 2, w1[:7], w2), lambda: g.expert_layer(x, logits, 2, w1[0], w2),
                 lambda: g.expert_layer(x.cpu(), logits, 2, w1, w2), lambda: g.expert_layer(x, logits, 2, w1.int(), w2)):
        with pytest.raises(ValueError):
            call()
    q1, s1 = g.quantise_blocks(w1, 128)
    q2, s2 = g.quantise_blocks(w2, 128)
    for call in (lambda: g.expert_layer(x, logits, 9, w1, w2), lambda: g.expert_layer(x, logits[:3], 2, w1, w2),
                 lambda: g.expert_layer(x, logits, 2, w1.half(), w2.half()), lambda: g.expert_layer(x, logits, 2, w1[:, :63], w2),
                 lambda: g.expert_layer(x, logits, 2, q1, q2), lambda: g.expert_layer(x, logits, 2, q1, w2, w1_scale=s1),
                 lambda: g.expert_layer(x, logits, 2, w1, w2, w1_scale=s1, w2_scale=s2),
                 lambda: g.expert_layer(x, logits, 2, q1, q2, w1_scale=s1, w2_scale=s2.half()),
                 lambda: g.expert_layer(x.float(), logits, 2, w1.float(), w2.float()),
                 lambda: g.expert_layer(x, logits, 2, w1, w2, out_dtype=torch.float16),
                 lambda: g.expert_layer(x, logits, 2, *(g.quantise_rows(w)[0] for w in (w1, w2))),
                 lambda: g.expert_layer(x, logits, 2, g.quantise_rows(w1)[0], q2, w1_scale=g.quantise_rows(w1)[1], w2_scale=g.quantise_rows(w2)[1])):
        with pytest.raises(g.GmagnusError) as err:
            call()
        assert err.value.status == 1
    with pytest.raises(g.GmagnusError) as err:
        g.expert_layer(rand((65, 64), torch.bfloat16, 1), rand((65, 8), torch.float32, 2), 2, w1, w2)
    assert err.value.status == 6
    with pytest.raises(RuntimeError, match="expert_layer has no autograd formula"):
        g.expert_layer(x.clone().requires_grad_(), logits, 2, w1, w2).float().sum().backward()
