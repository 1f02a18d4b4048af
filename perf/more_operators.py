"""Timed cases of what stands around the routed expert products in a layer.

A gated layer of experts begins with the root-mean-square norm of its rows (with
the residual's addition), and its two grouped products meet in a gate,
silu(g) * u. Both hand rows on in 16 bits or in 8 bits with a scale for each 128
columns, and both have gradients. The products themselves are also there in 8-bit
integers with a scale for each row and each column, and for the few tokens of a
decoding step the whole layer, from the router's logits to the tokens' sums, is one
call. Sizes run from one token to a long prompt.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128          # values that share a scale in E4M3
FP8_MAX = 448.0      # largest finite value of float8_e4m3fn
INT8_MAX = 127.0
SCALE_MIN = 2.0 ** -126
EPS = 1e-6


def listed():
    return [
        # one token of a decoding step: the norm in 16 bits for the router, in 8 bits for the experts; latency only
        {"name": "norm_one_token", "op": "norm", "tokens": 1, "n": 4096, "dtype": "bfloat16", "residual": True,
         "quantise": True, "backward": False},
        # a long prompt on its way into 8-bit products
        {"name": "norm_prompt", "op": "norm", "tokens": 16384, "n": 4096, "dtype": "bfloat16", "residual": True,
         "quantise": True, "backward": False},
        # a training batch: the norm and its gradients
        {"name": "norm_train", "op": "norm", "tokens": 8192, "n": 4096, "dtype": "bfloat16", "residual": True,
         "quantise": False, "backward": True},
        # the rows of a small decoding batch between its two products
        {"name": "gate_decode", "op": "gate", "rows": 64, "n": 1536, "dtype": "bfloat16", "quantise": True,
         "backward": False},
        # a long prompt's rows between its two 8-bit products
        {"name": "gate_prompt", "op": "gate", "rows": 32768, "n": 2048, "dtype": "bfloat16", "quantise": True,
         "backward": False},
        # a training batch of odd size, with the gradient
        {"name": "gate_ragged", "op": "gate", "rows": 9001, "n": 1365, "dtype": "float16", "quantise": False,
         "backward": True},
        # a decoding batch in 8-bit integers: a few rows for each of many experts
        {"name": "int8_decode", "op": "int8", "tokens": 16, "experts": 64, "top_k": 4, "dtype": "bfloat16", "n": 2048,
         "k": 2048, "masked": False},
        # a long prompt in 8-bit integers, activations quantised on the way
        {"name": "int8_prompt", "op": "int8", "tokens": 8192, "experts": 16, "top_k": 2, "dtype": "bfloat16",
         "n": 4096, "k": 4096, "masked": False},
        # a prompt of odd size through odd-sized weights
        {"name": "int8_odd", "op": "int8", "tokens": 1000, "experts": 12, "top_k": 3, "dtype": "float16", "n": 1001,
         "k": 777, "masked": True},
        # the whole layer for a single token: nothing but the chosen experts' weights to read
        {"name": "layer_one_token", "op": "layer", "tokens": 1, "experts": 16, "top_k": 2, "dtype": "bfloat16",
         "hidden": 1024, "inner": 2048, "fp8": False, "normalise": True, "masked": False},
        # a decoding batch: most experts are reached, by a token or two each
        {"name": "layer_decode", "op": "layer", "tokens": 16, "experts": 64, "top_k": 4, "dtype": "bfloat16",
         "hidden": 2048, "inner": 1024, "fp8": False, "normalise": True, "masked": False},
        # a larger one with weights held in E4M3, a side that ends inside a block, padding tokens and closed experts
        {"name": "layer_fp8", "op": "layer", "tokens": 48, "experts": 64, "top_k": 6, "dtype": "bfloat16",
         "hidden": 2048, "inner": 1000, "fp8": True, "normalise": False, "masked": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, hi=4096):
    """A matrix's side: half of them multiples of 64, the others any number."""
    v = _log_int(rng, 64, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["norm", "norm", "gate", "gate", "int8", "int8", "layer", "layer", "layer"])
    while True:
        case = {"op": op, "dtype": rng.choice(["bfloat16", "float16"])}
        if op in ("norm", "gate"):
            case["tokens" if op == "norm" else "rows"] = rows = _log_int(rng, 1, 32768)
            case["n"] = _side(rng, 8192)
            if op == "norm":
                case["residual"] = rng.random() < 0.6
            case["backward"] = rng.random() < 0.4
            case["quantise"] = not case["backward"] and rng.random() < 0.6
            if rows * case["n"] > (1 << 25 if case["backward"] else 1 << 26):
                continue
            return case
        case["tokens"] = _log_int(rng, 1, 64 if op == "layer" else 16384)
        case["experts"] = _log_int(rng, 1, 256)
        case["top_k"] = rng.randint(1, min(8, case["experts"]))
        case["masked"] = rng.random() < 0.3
        rows = case["tokens"] * case["top_k"]
        if op == "int8":
            case["n"], case["k"] = _side(rng), _side(rng)
            if case["experts"] * case["n"] * case["k"] > 1 << 28 or rows * case["n"] * case["k"] > 2.7e11:
                continue
            return case
        case["hidden"], case["inner"] = _side(rng), _side(rng)
        case["fp8"], case["normalise"] = rng.random() < 0.4, rng.random() < 0.5
        if case["experts"] * case["hidden"] * case["inner"] * 3 > 1 << 29:
            continue
        if min(case["experts"], rows) * case["hidden"] * case["inner"] * 3 > 1 << 28:
            continue
        return case


# ------------------------------------------------------------------- inputs
def _randn(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, device="cuda", generator=gen).mul_(scale).to(dtype)


def _logits(case, gen):
    """A router's logits: some experts are liked more than others. Masked: the last tokens are padding and some
    experts are closed, by -inf."""
    t, e = case["tokens"], case["experts"]
    l = torch.randn(t, e, device="cuda", generator=gen) + 0.5 * torch.randn(e, device="cuda", generator=gen)
    if case["masked"]:
        l[t - t // 16:] = -math.inf
        l[:, 3::7] = -math.inf
    return l


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = getattr(torch, case["dtype"])
    op = case["op"]
    state = {"op": op, "backward": case.get("backward", False), "quantise": case.get("quantise", False)}
    if op == "norm":
        shape = (case["tokens"], case["n"])
        state["x"] = _randn(gen, shape, dtype)
        state["residual"] = _randn(gen, shape, dtype, 3.0) if case["residual"] else None
        state["weight"] = (1.0 + 0.2 * torch.randn(case["n"], device="cuda", generator=gen)).to(dtype)
        if state["backward"]:
            state["d_y"] = _randn(gen, shape, dtype)
            state["d_total"] = _randn(gen, shape, dtype) if case["residual"] else None
        return state
    if op == "gate":
        state["h"] = _randn(gen, (case["rows"], 2 * case["n"]), dtype)
        if state["backward"]:
            state["d_a"] = _randn(gen, (case["rows"], case["n"]), dtype)
        return state
    logits = _logits(case, gen)
    state["top_k"] = case["top_k"]
    if op == "int8":
        state["group_ptr"], state["token"], _ = _plain_route(logits, case["top_k"], True)
        state["x"] = _randn(gen, (case["tokens"], case["k"]), dtype)
        w = _randn(gen, (case["experts"], case["n"], case["k"]), torch.float32, case["k"] ** -0.5)
        state["wq"], state["w_scale"] = _plain_quantise_rows(w)
        return state
    state["logits"], state["normalise"] = logits, case["normalise"]
    d, f, e = case["hidden"], case["inner"], case["experts"]
    state["x"] = _randn(gen, (case["tokens"], d), dtype)
    state["scales"] = None
    if case["fp8"]:
        state["w1"], s1 = _plain_quantise(_randn(gen, (e, 2 * f, d), torch.float32, d ** -0.5), BLOCK)
        state["w2"], s2 = _plain_quantise(_randn(gen, (e, d, f), torch.float32, f ** -0.5), BLOCK)
        state["scales"] = (s1, s2)
    else:
        state["w1"] = _randn(gen, (e, 2 * f, d), dtype, d ** -0.5)
        state["w2"] = _randn(gen, (e, d, f), dtype, f ** -0.5)
    return state


# --------------------------------------------------------------- plain forms
def _in_blocks(x, rows):
    """x padded with zeros to whole blocks, as [..., row blocks, rows, column blocks, BLOCK]."""
    n, k = x.shape[-2:]
    x = torch.nn.functional.pad(x, (0, -k % BLOCK, 0, -n % rows))
    return x.reshape(x.shape[:-2] + (x.shape[-2] // rows, rows, x.shape[-1] // BLOCK, BLOCK))


def _plain_quantise(x, rows):
    """float8_e4m3fn values and a scale for each block of `rows` x 128: its largest magnitude over 448."""
    n, k = x.shape[-2:]
    b = _in_blocks(x.float(), rows)
    scale = (b.abs().amax((-3, -1)) / FP8_MAX).clamp(min=SCALE_MIN)
    q = (b / scale[..., :, None, :, None]).clamp(-FP8_MAX, FP8_MAX)
    q = q.reshape(x.shape[:-2] + (b.shape[-4] * rows, b.shape[-2] * BLOCK))[..., :n, :k]
    return q.to(torch.float8_e4m3fn).contiguous(), scale


def _plain_values(q, scale, rows):
    n, k = q.shape[-2:]
    b = _in_blocks(q.float(), rows) * scale[..., :, None, :, None]
    return b.reshape(q.shape[:-2] + (b.shape[-4] * rows, b.shape[-2] * BLOCK))[..., :n, :k]


def _plain_quantise_rows(x):
    """int8 values and a scale for each row: its largest magnitude over 127."""
    scale = (x.float().abs().amax(-1) / INT8_MAX).clamp(min=SCALE_MIN)
    return torch.round(x.float() / scale[..., None]).clamp(-INT8_MAX, INT8_MAX).to(torch.int8), scale


def _plain_norm(s):
    x = s["x"]
    total = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    h = total.float()
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    y = h * r * s["weight"].float()
    out = [y.to(x.dtype)] + ([] if s["residual"] is None else [total])
    if s["quantise"]:
        out += list(_plain_quantise(y, 1))
    if s["backward"]:
        d, xhat = s["d_y"].float(), h * r
        g = d * s["weight"].float()
        d_x = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["d_total"] is not None:
            d_x = d_x + s["d_total"].float()
        out += [d_x.to(x.dtype), (d * xhat).sum(0)]
    return out


def _plain_gate(s):
    h = s["h"].float()
    n = h.shape[1] // 2
    g, u = h[:, :n], h[:, n:]
    sig = 1.0 / (1.0 + torch.exp(-g))
    a = g * sig * u
    out = [a.to(s["h"].dtype)]
    if s["quantise"]:
        out = list(_plain_quantise(a, 1))
    if s["backward"]:
        d = s["d_a"].float()
        out.append(torch.cat((d * u * sig * (1.0 + g * (1.0 - sig)), d * g * sig), 1).to(s["h"].dtype))
    return out


def _plain_route(logits, top_k, normalise):
    """The top_k largest logits of each row (ties: the lowest expert; -inf and NaN are never chosen): where each expert's
    entries begin, their tokens and softmax weights, expert by expert. Places past the last entry hold -1, weight 0."""
    t, e = logits.shape
    l = logits.float()
    l = torch.where(torch.isnan(l), -math.inf, l)
    best = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :top_k]
    chosen = torch.zeros(t, e, dtype=torch.bool, device=l.device).scatter_(1, best, True) & (l > -math.inf)
    top = l.amax(1, keepdim=True)
    p = torch.exp(l - torch.where(top == -math.inf, 0.0, top))
    p = p / (p * chosen if normalise else p).sum(1, keepdim=True)
    group_ptr = torch.zeros(e + 1, dtype=torch.int64, device=l.device)
    group_ptr[1:] = torch.cumsum(chosen.sum(0), 0)
    by_expert = chosen.t().nonzero()
    n = by_expert.shape[0]
    token = torch.full((t * top_k,), -1, dtype=torch.int32, device=l.device)
    token[:n] = by_expert[:, 1].to(torch.int32)
    weight = torch.zeros(t * top_k, device=l.device)
    weight[:n] = p.t()[chosen.t()]
    return group_ptr, token, weight


def _by_group(group_ptr, n_rows):
    """Each group's rows side by side, as many as the longest has: their numbers, and which of them there are."""
    cap = max(1, int((group_ptr[1:] - group_ptr[:-1]).max()))
    at = group_ptr[:-1, None] + torch.arange(cap, device=group_ptr.device)
    there = at < group_ptr[1:, None]
    return at.clamp(max=n_rows - 1), there


def _plain_int8(s):
    q, scale = _plain_quantise_rows(s["x"])
    n_rows = s["token"].numel()
    at, there = _by_group(s["group_ptr"], n_rows)
    x = q.float() * scale[:, None]
    rows = torch.where(there[..., None], x[s["token"][at].clamp(min=0).long()], 0.0)
    y = rows @ (s["wq"].float() * s["w_scale"][..., None]).transpose(1, 2)
    out = torch.zeros(n_rows, y.shape[2], dtype=s["x"].dtype, device=x.device)
    out[at[there]] = y[there].to(out.dtype)
    return out


def _plain_layer(s):
    x = s["x"]
    group_ptr, token, weight = _plain_route(s["logits"], s["top_k"], s["normalise"])
    at, there = _by_group(group_ptr, token.numel())
    used = there[:, 0].nonzero()[:, 0]  # the experts that a token has chosen
    at, there = at[used], there[used]
    if s["scales"] is None:
        w1, w2 = s["w1"][used].float(), s["w2"][used].float()
    else:
        w1 = _plain_values(s["w1"].view(torch.uint8)[used].view(torch.float8_e4m3fn), s["scales"][0][used], BLOCK)
        w2 = _plain_values(s["w2"].view(torch.uint8)[used].view(torch.float8_e4m3fn), s["scales"][1][used], BLOCK)
    n = w2.shape[2]
    rows = torch.where(there[..., None], x.float()[token[at].clamp(min=0).long()], 0.0)
    h = rows @ w1.transpose(1, 2)
    g, u = h[..., :n], h[..., n:]
    y = (g / (1.0 + torch.exp(-g)) * u) @ w2.transpose(1, 2) * weight[at][..., None]
    out = torch.zeros(x.shape[0], y.shape[2], device=x.device)
    return out.index_add_(0, token[at[there]].long(), y[there]).to(x.dtype)


# ---------------------------------------------------------------------- run
def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "gate": _plain_gate, "int8": _plain_int8, "layer": _plain_layer}[s["op"]](s)


def _run_own(s):
    from paper_2607_22866_amd import gmagnus as g

    fmt = torch.float8_e4m3fn if s["quantise"] else None
    if s["op"] == "norm":
        r = g.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, quantise=fmt, plain=True)
        out = [r.y] + ([] if s["residual"] is None else [r.total])
        if s["quantise"]:
            out += [r.q, r.scale]
        if s["backward"]:
            total = s["x"] if s["residual"] is None else r.total
            out += list(g.rms_norm_backward(total, s["weight"], s["d_y"], d_total=s["d_total"], eps=EPS))
        return out
    if s["op"] == "gate":
        r = g.gate(s["h"], quantise=fmt)
        out = [r.q, r.scale] if s["quantise"] else [r.y]
        if s["backward"]:
            out.append(g.gate_backward(s["h"], s["d_a"]))
        return out
    if s["op"] == "int8":
        q, scale = g.quantise_rows(s["x"])
        return g.group_product_int8(q, scale, s["wq"], s["w_scale"], s["group_ptr"], index=s["token"],
                                    out_dtype=s["x"].dtype)
    s1, s2 = s["scales"] or (None, None)
    return g.expert_layer(s["x"], s["logits"], s["top_k"], s["w1"], s["w2"], normalise=s["normalise"], w1_scale=s1,
                          w2_scale=s2)


# ---------------------------------------------------------------------- work
def work(case):
    """Inputs read once, outputs written once. Weights count for the experts that uniform choices would reach."""
    if case["op"] == "norm":
        t, n = case["tokens"], case["n"]
        streams = 2 + 2 * case["residual"]  # x and y, the residual and the sum
        if case["backward"]:  # the gradients of y and of x, and of the sum (which is read again in a call of its own)
            streams += 3 + case["residual"]
        byts = t * n * 2 * streams + 2 * n
        if case["quantise"]:
            byts += t * (n + 4 * -(-n // BLOCK))
        if case["backward"]:
            byts += 6 * n
        return {"bytes": float(byts), "flops": float((4 + 9 * case["backward"]) * t * n)}
    if case["op"] == "gate":
        t, n = case["rows"], case["n"]
        byts = 4 * t * n + (t * (n + 4 * -(-n // BLOCK)) if case["quantise"] else 2 * t * n)
        if case["backward"]:  # h once more, the gradients of a and of h
            byts += 10 * t * n
        return {"bytes": float(byts), "flops": float((6 + 12 * case["backward"]) * t * n)}
    t, e, k = case["tokens"], case["experts"], case["top_k"]
    closed = len(range(3, e, 7)) if case["masked"] else 0
    live_t = t - t // 16 if case["masked"] else t
    rows = live_t * min(k, e - closed)
    reached = (e - closed) * (1.0 - (1.0 - min(1.0, k / max(1, e - closed))) ** live_t)
    if case["op"] == "int8":
        n, kk = case["n"], case["k"]
        byts = t * kk * 2 + t * k * (2 * n + 4) + reached * (n * kk + 4 * n)
        return {"bytes": float(byts), "flops": 2.0 * rows * n * kk}
    d, f = case["hidden"], case["inner"]
    byts = 4 * t * d + 4 * t * e + reached * 3 * d * f * (1 if case["fp8"] else 2)
    return {"bytes": float(byts), "flops": 6.0 * rows * d * f}


# --------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in 64 bits; the products expert by expert."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "gate":
        g, u = s["h"].double().chunk(2, 1)
        sig = torch.sigmoid(g)
        if s["quantise"]:
            return _exact_quantise(g * sig * u)
        out = [g * sig * u]
        if s["backward"]:
            d = s["d_a"].double()
            out.append(torch.cat((d * u * (sig + g * sig * torch.sigmoid(-g)), d * (g * sig)), 1))
        return out
    if case["op"] == "int8":
        x = s["x"].double()
        scale = (x.abs().max(1).values / INT8_MAX).clamp_min(SCALE_MIN)
        x = torch.round(x / scale[:, None]) * scale[:, None]
        gp, token = s["group_ptr"].tolist(), s["token"].long()
        y = torch.zeros(token.numel(), case["n"], dtype=torch.float64, device="cuda")
        for e in range(len(gp) - 1):
            if gp[e] < gp[e + 1]:
                w = s["wq"][e].double() * s["w_scale"][e].double()[:, None]
                y[gp[e]:gp[e + 1]] = x[token[gp[e]:gp[e + 1]]].matmul(w.t())
        return y
    return _exact_layer(case, s)


def _exact_quantise(y):
    """[values on the grid of float8_e4m3fn, scales]."""
    kb = -(-y.shape[1] // BLOCK)
    q, scale = torch.zeros_like(y), torch.zeros(y.shape[0], kb, dtype=torch.float64, device="cuda")
    for b in range(kb):
        part = y[:, b * BLOCK:(b + 1) * BLOCK]
        scale[:, b] = (part.abs().max(1).values / FP8_MAX).clamp_min(SCALE_MIN)
        q[:, b * BLOCK:(b + 1) * BLOCK] = (part / scale[:, b:b + 1]).float().to(torch.float8_e4m3fn).double()
    return [q, scale]


def _exact_norm(s):
    x, w = s["x"].double(), s["weight"].double()
    out_total = []
    if s["residual"] is not None:
        x = (x + s["residual"].double()).to(s["x"].dtype).double()
        out_total = [x]
    root = torch.sqrt(x.pow(2).sum(1, keepdim=True) / x.shape[1] + EPS)
    y = x / root * w
    out = [y] + out_total
    if s["quantise"]:
        out += _exact_quantise(y)
    if s["backward"]:
        d = s["d_y"].double()
        g = d * w
        d_x = g / root - x * (g * x).sum(1, keepdim=True) / (x.shape[1] * root.pow(3))
        if s["d_total"] is not None:
            d_x += s["d_total"].double()
        out += [d_x, (d * x / root).sum(0)]
    return out


def _exact_layer(case, s):
    l = s["logits"].double()
    t, e = l.shape
    left, chosen = l.clone(), torch.zeros(t, e, dtype=torch.bool, device="cuda")
    rows = torch.arange(t, device="cuda")
    for _ in range(case["top_k"]):
        top = left.max(1, keepdim=True).values
        first = torch.where((left == top) & (top > -math.inf), torch.arange(e, device="cuda"), e).min(1).values
        ok = first < e
        chosen[rows[ok], first[ok]] = True
        left[rows[ok], first[ok]] = -math.inf
    z = torch.exp(l - l.max(1, keepdim=True).values).nan_to_num(0.0)
    p = (z / (z * chosen if s["normalise"] else z).sum(1, keepdim=True)).nan_to_num(0.0)
    d, f = case["hidden"], case["inner"]
    x, out = s["x"].double(), torch.zeros(t, d, dtype=torch.float64, device="cuda")

    def weights(w, scale, i):
        w = w[i].double()
        if scale is None:
            return w
        up, across = (torch.arange(v, device="cuda") // BLOCK for v in w.shape)
        return w * scale[i].double()[up][:, across]

    s1, s2 = s["scales"] or (None, None)
    for i in chosen.any(0).nonzero()[:, 0].tolist():
        mine = chosen[:, i]
        h = x[mine].matmul(weights(s["w1"], s1, i).t())
        a = h[:, :f] * torch.sigmoid(h[:, :f]) * h[:, f:]
        out[mine] += p[mine, i, None] * a.matmul(weights(s["w2"], s2, i).t())
    return out
