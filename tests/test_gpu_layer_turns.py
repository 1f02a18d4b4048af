"""What a kernel does in its second turn and later: the layer's items beyond its grid, rows to 8-bit integers beyond
theirs. And the layer's weights in integers at other strides, alignments and far offsets."""
import pytest

from tests import rows_ref as rr
from tests.test_gpu_expert_layer_few import case, check, rand

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def g():
    from paper_2607_22866_amd import gmagnus

    gmagnus.load()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return gmagnus


# tokens, experts, top_k, hidden, inner, outputs: 1250 to 9000 items of 16 gates, of which a launch's work groups take
# 1024 at a time; experts of a few rows, of more than 16 and of more than 32
TURNS = [(16, 64, 4, 200, 1000, 64), (16, 3, 3, 130, 9001, 40), (48, 64, 6, 136, 1000, 40), (64, 4, 3, 80, 5000, 24), (40, 200, 8, 64, 520, 96)]


@pytest.mark.parametrize("t,e,k,d,f,n", TURNS)
@pytest.mark.parametrize("kind", ["16 bits", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_more_items_than_work_groups(g, t, e, k, d, f, n, kind, dtype):
    x, logits, w1, w2 = case(t, e, d, f, n, dtype, fp8=kind != "16 bits")
    s1 = s2 = None
    if kind == "e4m3":
        (w1, s1), (w2, s2) = g.quantise_blocks(w1, 128), g.quantise_blocks(w2, 128)
    elif kind == "int8":
        (w1, s1), (w2, s2) = g.quantise_rows(w1), g.quantise_rows(w2)
    used = int((g.route(logits, k).group_ptr.diff() > 0).sum())
    assert used * -(-f // 16) > 1200
    check(g, x, logits, k, w1, w2, s1=s1, s2=s2, out_dtype=torch.float32)
    y = check(g, x, logits, k, w1, w2, s1=s1, s2=s2, normalise=False)
    assert torch.equal(y, g.expert_layer(x, logits, k, w1, w2, w1_scale=s1, w2_scale=s2, normalise=False))


# rows of a turn: 8192 up to 1024 columns, 2048 above
@pytest.mark.parametrize("shape", [(8200, 40), (20011, 513), (2100, 2056), (4300, 1100), (2050, 8195), (3, 2900, 40), (5, 900, 1032), (70, 61, 1025)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_to_integers_beyond_a_turn(g, shape, dtype):
    x = rand(shape, dtype, sum(shape), 5.0)
    # every row has a size of its own
    x *= (1 + torch.arange(x[..., 0].numel(), device="cuda").reshape(x.shape[:-1]) % 97)[..., None].to(dtype) / 64
    q, s = g.quantise_rows(x)
    n = shape[-1]
    want = x.double().cpu().reshape(-1, n)
    rr.check_int8(q.cpu().reshape(-1, n), s.cpu().flatten(), want, torch.zeros_like(want))


@pytest.mark.parametrize("off", [1, 3, 8, 16])
@pytest.mark.parametrize("tokens", [5, 19])
def test_integers_at_other_strides(g, off, tokens):
    x, logits, w1, w2 = case(tokens, 6, 300 + off, 130 + off, 90 + off, torch.bfloat16, fp8=True)
    (w1, s1), (w2, s2) = g.quantise_rows(w1), g.quantise_rows(w2)
    s1, s2 = torch.cat((s1, s1), 1)[:, 5:265], s2[:, off:]
    x, logits, w1, w2 = x[:, off:], torch.cat((logits, logits), 1)[:, 3:9], w1[:, :260, off:], w2[:, off:, off:]
    buf = torch.full((tokens, 90 + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    a = check(g, x, logits, 2, w1, w2, s1=s1, s2=s2, out=buf[:, 3:93])
    b = g.expert_layer(*(v.contiguous() for v in (x, logits)), 2, w1.contiguous(), w2.contiguous(), w1_scale=s1.contiguous(), w2_scale=s2.contiguous())
    assert torch.equal(a, b) and bool((buf[:, :3] == 5).all()) and bool((buf[:, 93:] == 5).all())


@pytest.mark.parametrize("tokens", [3, 20])
def test_integers_past_32_bit_offsets(g, tokens):
    # two experts more than 2^32 bytes apart, and their scales more than 2^32 bytes
    x, logits, w1, w2 = case(tokens, 2, 64, 32, 48, torch.bfloat16, fp8=True)
    (w1, s1), (w2, s2) = g.quantise_rows(w1), g.quantise_rows(w2)
    big = torch.zeros((2, (1 << 32) + 8192), dtype=torch.int8, device="cuda")
    v1, v2 = big[:, :64 * 64].unflatten(1, (64, 64)), big[:, 4096:4096 + 48 * 32].unflatten(1, (48, 32))
    far = torch.zeros((2, (1 << 30) + 256), device="cuda")
    f1, f2 = far[:, :64], far[:, 64:112]
    for to, of in ((v1, w1), (v2, w2), (f1, s1), (f2, s2)):
        to.copy_(of)
    assert torch.equal(g.expert_layer(x, logits, 2, v1, v2, w1_scale=f1, w2_scale=f2), g.expert_layer(x, logits, 2, w1, w2, w1_scale=s1, w2_scale=s2))
