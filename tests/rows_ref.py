"""64-bit forms of what happens to rows around the products (torch, on the host), for the tests, and how far
results in fewer bits may be from them.

Roundings are counted: half a step of the result's type once, and half a step of
fp32 (2^-24, relative) for every operation on the way to it. A row's sum of
squares (or of products) is made of at most 16 terms a lane in turn (longer rows: one
more for every 8192 columns, and 8), six steps over a wave and 16 over the waves: sum_steps()."""
import torch

BLOCK = 128
U32 = 2.0 ** -24
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}  # a subnormal's step


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def sum_steps(n):
    return 16 + n // 8192 + 8 + 6 + 16


def rms_norm(total, weight, eps):
    h = total.double()
    r = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    return h * r * (1.0 if weight is None else weight.double())


def rms_norm_error(y, n):
    """The sum's roundings count half under the root; six operations make the root and the result."""
    return (0.5 * sum_steps(n) + 6) * U32 * y.abs()


def rms_norm_backward(total, weight, d_y, d_total, eps):
    """(d_x, its sum of magnitudes, d_weight, its sum of magnitudes)."""
    h, d = total.double(), d_y.double()
    r = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    g = d * (1.0 if weight is None else weight.double())
    dt = torch.zeros_like(h) if d_total is None else d_total.double()
    d_x = r * (g - h * r * r * (g * h).mean(1, keepdim=True)) + dt
    mag = r * (g.abs() + h.abs() * r * r * (g * h).abs().mean(1, keepdim=True)) + dt.abs()
    return d_x, mag, (d * h * r).sum(0), (d * h * r).abs().sum(0)


def backward_error(mag, n):
    """Two sums over the row (the squares' counts three halves of times through r^3) and ten operations."""
    return (2.5 * sum_steps(n) + 10) * U32 * mag


def weight_error(mag, t, n):
    """Rows of a unit in turn (512 units at most, four waves each), 32 units in turn, 16 waves; r's and two more roundings."""
    return (t / 512 + 4 + 32 + 16 + 0.5 * sum_steps(n) + 8) * U32 * mag


def gate(h):
    g, u = h.double().chunk(2, 1)
    return g * torch.sigmoid(g) * u


def gate_error(y, h):
    """sigma: a few units for e^x (8 counted), two operations, then two products; e^x is zero below 2^-126."""
    g, u = h.double().chunk(2, 1)
    return 12 * U32 * y.abs() + 2.0 ** -125 * (1 + (g * u).abs())


def gate_backward(h, d_y):
    """(d_h, its sum of magnitudes)."""
    g, u = h.double().chunk(2, 1)
    d, s, rest = d_y.double(), torch.sigmoid(g), torch.sigmoid(-g)
    one = torch.cat((d * u * s * (1 + g * rest), d * g * s), 1)
    return one, torch.cat(((d * u).abs() * s * (1 + g.abs() * rest), (d * g).abs() * s), 1)


def gate_backward_error(mag, h, d_y):
    """As gate_error with five more operations. e^x is zero below 2^-126, which takes at most that from sigma (x below
    -87) and so |d_y u| (1 + |g|) or |d_y g| times that from the results."""
    g, u = h.double().chunk(2, 1)
    d = d_y.double()
    lost = torch.cat(((d * u).abs() * (1 + g.abs()), (d * g).abs()), 1)
    return 20 * U32 * mag + 2.0 ** -125 * (1 + lost)


def check_e4m3(q, scale, want, error):
    """Blocks of 128 of the 64-bit `want`, which the values before rounding are within `error` of."""
    n = want.shape[1]
    pad = -n % BLOCK
    blocks = torch.nn.functional.pad(want.abs(), (0, pad)).unflatten(1, (-1, BLOCK))
    slack = torch.nn.functional.pad(error, (0, pad)).unflatten(1, (-1, BLOCK)).amax(2)
    top = (blocks.amax(2) / 448.0).clamp(min=2.0 ** -126)
    assert scale.dtype == torch.float32 and q.dtype == torch.float8_e4m3fn
    assert bool(((scale.double() - top).abs() <= slack / 448 + U32 * top).all())
    s = scale.double().repeat_interleave(BLOCK, 1)[:, :n]
    # half a step of three bits, of a subnormal 2^-10 of the scale; the quotient's rounding moves a value across
    # a border by no more than itself
    off = 2.0 ** -4 * want.abs() + 2.0 ** -10 * s + 2 * error + 2 * U32 * want.abs()
    assert bool(((q.double() * s - want).abs() <= off).all())


def check_int8(q, scale, want, error):
    top = (want.abs().amax(1) / 127.0).clamp(min=2.0 ** -126)
    assert scale.dtype == torch.float32 and q.dtype == torch.int8
    assert bool(((scale.double() - top).abs() <= error.amax(1) / 127 + U32 * top).all())
    s = scale.double()[:, None]
    off = 0.5 * s + 2 * error + 128 * 2 * U32 * s
    assert bool(((q.double() * s - want).abs() <= off).all())
    assert bool((q.int().abs() <= 127).all())
    full = want.abs().amax(1) > 2.0 ** -118
    assert bool((q.int().abs().amax(1)[full] == 127).all())
