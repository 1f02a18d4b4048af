"""Timed cases of the routed expert products.

A layer of experts is a sparse matrix product: the routing matrix R (tokens x
experts, a few entries a row) says which rows meet which expert's weights. The
cases cover what a program calls for such a layer: the routing matrix from a
router's logits, in both orders (and the logits' gradient), the products
grouped by expert with ragged sizes in 16 bits and in 8 bits with a scale for
each block of 128, their gradients, and the weighted sum of a token's results
(and its gradients). Sizes run from one token to a long prompt.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128          # values that share a scale
FP8_MAX = 448.0      # largest finite value of float8_e4m3fn
SCALE_MIN = 2.0 ** -126


def listed():
    return [
        # one token of a decoding step asks the router: launches and latency only
        {"name": "route_one_token", "op": "route", "tokens": 1, "experts": 64, "top_k": 4, "dtype": "float32",
         "normalise": True, "backward": False, "masked": False},
        # a long prompt or a training batch through a wide router, padding tokens masked out, with the logits' gradient
        {"name": "route_train", "op": "route", "tokens": 16384, "experts": 256, "top_k": 8, "dtype": "bfloat16",
         "normalise": False, "backward": True, "masked": True},
        # the results of a small decoding batch summed per token
        {"name": "combine_decode", "op": "combine", "tokens": 16, "experts": 64, "top_k": 4, "dtype": "bfloat16",
         "n": 2048, "backward": False, "masked": False},
        # a training batch: the sum and its gradients
        {"name": "combine_train", "op": "combine", "tokens": 8192, "experts": 32, "top_k": 4, "dtype": "bfloat16",
         "n": 4096, "backward": True, "masked": False},
        # a single token's products: nothing but the chosen experts' weights to read
        {"name": "product_one_token", "op": "product", "tokens": 1, "experts": 16, "top_k": 2, "dtype": "bfloat16",
         "n": 1024, "k": 2048, "masked": False},
        # a decoding batch: a few rows for each of many experts
        {"name": "product_decode", "op": "product", "tokens": 16, "experts": 64, "top_k": 4, "dtype": "bfloat16",
         "n": 2048, "k": 2048, "masked": False},
        # a prompt of odd size through odd-sized weights
        {"name": "product_odd", "op": "product", "tokens": 1531, "experts": 12, "top_k": 3, "dtype": "float16",
         "n": 1001, "k": 777, "masked": True},
        # a long prompt: the products are bound by the matrix units
        {"name": "product_prompt", "op": "product", "tokens": 8192, "experts": 32, "top_k": 4, "dtype": "bfloat16",
         "n": 2048, "k": 4096, "masked": False},
        # the training step's two products of the gradient
        {"name": "gradients_train", "op": "gradients", "tokens": 4096, "experts": 16, "top_k": 4,
         "dtype": "bfloat16", "n": 2048, "k": 2048, "masked": False},
        # a small ragged training batch with padding tokens and experts that get nothing
        {"name": "gradients_ragged", "op": "gradients", "tokens": 1000, "experts": 40, "top_k": 2,
         "dtype": "float16", "n": 776, "k": 1290, "masked": True},
        # decoding with weights held in 8 bits
        {"name": "fp8_decode", "op": "fp8", "tokens": 4, "experts": 32, "top_k": 2, "dtype": "bfloat16", "n": 2048,
         "k": 4096, "masked": False},
        # a long prompt with weights held in 8 bits, activations quantised on the way
        {"name": "fp8_prompt", "op": "fp8", "tokens": 8192, "experts": 16, "top_k": 2, "dtype": "bfloat16",
         "n": 4096, "k": 4096, "masked": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng):
    """A weight's side: half of them multiples of 64, the others any number."""
    v = _log_int(rng, 64, 4096)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["route", "combine", "product", "product", "gradients", "gradients", "fp8", "fp8"])
    while True:
        case = {"op": op, "tokens": _log_int(rng, 1, 16384), "experts": _log_int(rng, 1, 256)}
        case["top_k"] = rng.randint(1, min(8, case["experts"]))
        case["dtype"] = rng.choice(["bfloat16", "float16"])
        if op == "route":
            case["dtype"] = rng.choice(["float32", "bfloat16", "float16"])
            case["normalise"] = rng.random() < 0.5
        if op in ("route", "combine"):
            case["backward"] = rng.random() < 0.5
        if op == "combine":
            case["n"] = _side(rng)
        if op in ("product", "gradients", "fp8"):
            case["n"], case["k"] = _side(rng), _side(rng)
        case["masked"] = rng.random() < 0.3
        rows = case["tokens"] * case["top_k"]
        if op == "combine" and rows * case["n"] > 1 << 27:
            continue
        if op in ("product", "gradients", "fp8"):
            passes = 2 if op == "gradients" else 1
            if case["experts"] * case["n"] * case["k"] > 1 << 28 or passes * rows * case["n"] * case["k"] > 2.7e11:
                continue
        return case


# ------------------------------------------------------------------- inputs
def _logits(case, gen):
    """A router's logits: some experts are liked more than others. Masked: the last tokens are padding and some
    experts are closed, by -inf."""
    t, e = case["tokens"], case["experts"]
    l = torch.randn(t, e, device="cuda", generator=gen) + 0.5 * torch.randn(e, device="cuda", generator=gen)
    if case["masked"]:
        l[t - t // 16:] = -math.inf
        l[:, 3::7] = -math.inf
    return l


def _randn(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, device="cuda", generator=gen).mul_(scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = getattr(torch, case["dtype"])
    logits = _logits(case, gen)
    state = {"op": case["op"], "top_k": case["top_k"], "backward": case.get("backward", False)}
    if case["op"] == "route":
        state["logits"] = logits.to(dtype)
        state["normalise"] = case["normalise"]
        state["d_weight"] = _randn(gen, (case["tokens"] * case["top_k"],), torch.float32)
        return state
    row_ptr, _, weight, group_ptr, token, slot, _ = _plain_route(logits, case["top_k"], True)
    state.update(row_ptr=row_ptr, weight=weight, group_ptr=group_ptr, token=token, slot=slot)
    rows = case["tokens"] * case["top_k"]
    if case["op"] == "combine":
        state["y"] = _randn(gen, (rows, case["n"]), dtype)
        state["d_out"] = _randn(gen, (case["tokens"], case["n"]), dtype)
        return state
    state["x"] = _randn(gen, (case["tokens"], case["k"]), dtype)
    w = _randn(gen, (case["experts"], case["n"], case["k"]), torch.float32, case["k"] ** -0.5)
    if case["op"] == "fp8":
        state["wq"], state["w_scale"] = _plain_quantise(w, BLOCK)
        state["dtype"] = dtype
    else:
        state["w"] = w.to(dtype)
    if case["op"] == "gradients":
        state["d_y"] = _randn(gen, (rows, case["n"]), dtype)
    return state


# --------------------------------------------------------------- plain forms
def _plain_route(logits, top_k, normalise):
    """The top_k largest logits of each row (ties: the lowest expert; -inf and NaN are never chosen), softmax weights,
    and the entries in both orders. Places past the last entry hold -1, weight 0."""
    t, e = logits.shape
    l = logits.float()
    l = torch.where(torch.isnan(l), -math.inf, l)
    best = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :top_k]
    chosen = torch.zeros(t, e, dtype=torch.bool, device=l.device).scatter_(1, best, True) & (l > -math.inf)
    top = l.amax(1, keepdim=True)
    p = torch.exp(l - torch.where(top == -math.inf, 0.0, top))
    p = p / (p * chosen if normalise else p).sum(1, keepdim=True)
    row_ptr = torch.zeros(t + 1, dtype=torch.int64, device=l.device)
    row_ptr[1:] = torch.cumsum(chosen.sum(1), 0)
    group_ptr = torch.zeros(e + 1, dtype=torch.int64, device=l.device)
    group_ptr[1:] = torch.cumsum(chosen.sum(0), 0)
    at = group_ptr[:-1] + torch.cumsum(chosen, 0) - 1
    by_token, by_expert = chosen.nonzero(), chosen.t().nonzero()
    n = by_token.shape[0]

    def whole(v, dtype, empty):
        out = torch.full((t * top_k,), empty, dtype=dtype, device=l.device)
        out[:n] = v.to(dtype)
        return out

    return (row_ptr, whole(by_token[:, 1], torch.int32, -1), whole(p[chosen], torch.float32, 0), group_ptr,
            whole(by_expert[:, 1], torch.int32, -1), whole(at[chosen], torch.int32, -1),
            whole(p.t()[chosen.t()], torch.float32, 0))


def _plain_route_backward(logits, row_ptr, expert, weight, d_weight, normalise):
    t, e = logits.shape
    n = int(row_ptr[-1])
    row = torch.repeat_interleave(torch.arange(t, device=logits.device), row_ptr[1:] - row_ptr[:-1])
    place = (row, expert[:n].long())
    zero = torch.zeros(t, e, device=logits.device)
    g = zero.index_put(place, d_weight[:n])
    if normalise:
        p = zero.index_put(place, weight[:n])
    else:
        l = logits.float()
        l = torch.where(torch.isnan(l), -math.inf, l)
        top = l.amax(1, keepdim=True)
        p = torch.exp(l - torch.where(top == -math.inf, 0.0, top))
        p = p / p.sum(1, keepdim=True)
        p = torch.where(top == -math.inf, 0.0, p)
    return (p * (g - (p * g).sum(1, keepdim=True))).to(logits.dtype)


def _by_group(group_ptr, n_rows):
    """Each group's rows side by side, as many as the longest has: their numbers, and which of them there are."""
    cap = max(1, int((group_ptr[1:] - group_ptr[:-1]).max()))
    at = group_ptr[:-1, None] + torch.arange(cap, device=group_ptr.device)
    there = at < group_ptr[1:, None]
    return at.clamp(max=n_rows - 1), there


def _pick(x, at, there, index=None):
    at = at if index is None else index[at].clamp(min=0).long()
    return torch.where(there[..., None], x.float()[at], 0.0)


def _plain_product(x, w, group_ptr, index, n_rows, dtype):
    """Row r of group e: x[index[r]] times the rows of w[e]."""
    at, there = _by_group(group_ptr, n_rows)
    y = _pick(x, at, there, index) @ w.float().transpose(1, 2)
    out = torch.zeros(n_rows, w.shape[1], dtype=dtype, device=x.device)
    out[at[there]] = y[there].to(dtype)
    return out


def _plain_gradients(d_y, x, w, group_ptr, index):
    at, there = _by_group(group_ptr, d_y.shape[0])
    d = _pick(d_y, at, there)
    d_x = torch.zeros(d_y.shape[0], w.shape[2], dtype=x.dtype, device=x.device)
    d_x[at[there]] = (d @ w.float())[there].to(x.dtype)
    return d_x, (d.transpose(1, 2) @ _pick(x, at, there, index)).to(w.dtype)


def _entries(row_ptr, slot):
    k = slot.numel() // (row_ptr.numel() - 1)
    at = row_ptr[:-1, None] + torch.arange(k, device=slot.device)
    there = at < row_ptr[1:, None]
    at = at.clamp(max=slot.numel() - 1)
    return at, there, slot[at].clamp(min=0).long()


def _plain_combine(y, row_ptr, slot, weight):
    at, there, s = _entries(row_ptr, slot)
    return (y.float()[s] * torch.where(there, weight[at], 0.0)[..., None]).sum(1).to(y.dtype)


def _plain_combine_backward(y, row_ptr, slot, weight, d_out):
    at, there, s = _entries(row_ptr, slot)
    d = d_out.float()[:, None]
    d_y = torch.zeros_like(y)
    d_y[s[there]] = (weight[at][..., None] * d)[there].to(y.dtype)
    d_weight = torch.zeros_like(weight)
    d_weight[at[there]] = (y.float()[s] * d).sum(-1)[there]
    return d_y, d_weight


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


# ---------------------------------------------------------------------- run
def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "route":
        r = _plain_route(s["logits"], s["top_k"], s["normalise"])
        if s["backward"]:
            r += (_plain_route_backward(s["logits"], r[0], r[1], r[2], s["d_weight"], s["normalise"]),)
        return r
    if s["op"] == "combine":
        out = _plain_combine(s["y"], s["row_ptr"], s["slot"], s["weight"])
        if s["backward"]:
            return (out,) + _plain_combine_backward(s["y"], s["row_ptr"], s["slot"], s["weight"], s["d_out"])
        return out
    if s["op"] == "product":
        return _plain_product(s["x"], s["w"], s["group_ptr"], s["token"], s["token"].numel(), s["x"].dtype)
    if s["op"] == "gradients":
        return _plain_gradients(s["d_y"], s["x"], s["w"], s["group_ptr"], s["token"])
    q, scale = _plain_quantise(s["x"], 1)
    y = _plain_product(_plain_values(q, scale, 1), _plain_values(s["wq"], s["w_scale"], BLOCK), s["group_ptr"],
                       s["token"], s["token"].numel(), s["dtype"])
    return q, scale, y


def _run_own(s):
    from paper_2607_22866_amd import gmagnus as g

    if s["op"] == "route":
        r = g.route(s["logits"], s["top_k"], normalise=s["normalise"])
        out = (r.row_ptr, r.expert, r.weight, r.group_ptr, r.token, r.slot, r.group_weight)
        return out + (g.route_backward(s["logits"], r, s["d_weight"]),) if s["backward"] else out
    if s["op"] == "combine":
        out = g.combine(s["y"], s["row_ptr"], s["slot"], s["weight"])
        if s["backward"]:
            return (out,) + g.combine_backward(s["y"], s["row_ptr"], s["slot"], s["weight"], s["d_out"])
        return out
    if s["op"] == "product":
        return g.group_product(s["x"], s["w"], s["group_ptr"], index=s["token"])
    if s["op"] == "gradients":
        return (g.group_product(s["d_y"], s["w"], s["group_ptr"], transposed=True),
                g.group_outer(s["d_y"], s["x"], s["group_ptr"], index=s["token"]))
    q, scale = g.quantise_blocks(s["x"])
    return q, scale, g.group_product_fp8(q, scale, s["wq"], s["w_scale"], s["group_ptr"], index=s["token"],
                                         out_dtype=s["dtype"])


# ---------------------------------------------------------------------- work
def work(case):
    """Inputs read once, outputs written once. Weights count for the experts that uniform choices would reach."""
    t, e, k = case["tokens"], case["experts"], case["top_k"]
    size = 4 if case["dtype"] == "float32" else 2
    closed = len(range(3, e, 7)) if case["masked"] else 0
    live_t = t - t // 16 if case["masked"] else t
    rows = live_t * min(k, e - closed)
    if case["op"] == "route":
        byts = t * e * size + 8 * (t + 1) + 8 * (e + 1) + 20 * t * k
        if case["backward"]:
            byts += t * e * size + 4 * rows
        return {"bytes": float(byts), "flops": float((3 if case["backward"] else 1) * 2 * t * e)}
    if case["op"] == "combine":
        n = case["n"]
        byts = (rows + t) * n * size + 8 * rows + 8 * t
        flops = 2 * rows * n
        if case["backward"]:  # the results and the rows' gradient once more; the sum's gradient
            byts += (rows + t) * n * size + 4 * rows
            flops *= 2.5
        return {"bytes": float(byts), "flops": float(flops)}
    n, kk = case["n"], case["k"]
    reached = (e - closed) * (1.0 - (1.0 - min(1.0, k / max(1, e - closed))) ** live_t)
    if case["op"] == "product":
        byts = (t * kk + rows * n + reached * n * kk) * size
        return {"bytes": float(byts), "flops": 2.0 * rows * n * kk}
    if case["op"] == "gradients":
        byts = (t * kk + rows * (n + kk) + (reached + e) * n * kk) * size
        return {"bytes": float(byts), "flops": 4.0 * rows * n * kk}
    byts = t * kk * (size + 1) + rows * n * size + reached * n * kk
    return {"bytes": float(byts), "flops": 2.0 * rows * n * kk}


# --------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in 64 bits, expert by expert."""
    s = prepare(case, seed)
    if case["op"] == "route":
        return _exact_route(s)
    gp = s["group_ptr"].tolist()
    groups = range(len(gp) - 1)
    if case["op"] == "combine":
        return _exact_combine(s, case["backward"])
    token = s["token"].long()
    rows = token.numel()
    if case["op"] == "fp8":
        x = s["x"].double()
        kb = -(-x.shape[1] // BLOCK)
        q, scale = torch.zeros_like(x), torch.zeros(x.shape[0], kb, dtype=torch.float64, device="cuda")
        for b in range(kb):
            part = x[:, b * BLOCK:(b + 1) * BLOCK]
            scale[:, b] = (part.abs().max(1).values / FP8_MAX).clamp_min(SCALE_MIN)
            q[:, b * BLOCK:(b + 1) * BLOCK] = (part / scale[:, b:b + 1]).float().to(torch.float8_e4m3fn).double()
        spread = torch.arange(x.shape[1], device="cuda") // BLOCK
        x = q * scale[:, spread]
        y = torch.zeros(rows, case["n"], dtype=torch.float64, device="cuda")
        up = torch.arange(case["n"], device="cuda") // BLOCK
        for e in groups:
            if gp[e] < gp[e + 1]:
                w = s["wq"][e].double() * s["w_scale"][e].double()[up][:, spread]
                y[gp[e]:gp[e + 1]] = x[token[gp[e]:gp[e + 1]]].matmul(w.t())
        return q, scale, y
    x, w = s["x"].double(), s["w"]
    if case["op"] == "product":
        y = torch.zeros(rows, case["n"], dtype=torch.float64, device="cuda")
        for e in groups:
            if gp[e] < gp[e + 1]:
                y[gp[e]:gp[e + 1]] = x[token[gp[e]:gp[e + 1]]].matmul(w[e].double().t())
        return y
    d_x = torch.zeros(rows, case["k"], dtype=torch.float64, device="cuda")
    d_w = torch.zeros(w.shape, dtype=torch.float64, device="cuda")
    for e in groups:
        if gp[e] < gp[e + 1]:
            d = s["d_y"][gp[e]:gp[e + 1]].double()
            d_x[gp[e]:gp[e + 1]] = d.matmul(w[e].double())
            d_w[e] = d.t().matmul(x[token[gp[e]:gp[e + 1]]])
    return d_x, d_w


def _exact_route(s):
    l = s["logits"].double()
    t, e = l.shape
    k = s["top_k"]
    left, chosen = l.clone(), torch.zeros(t, e, dtype=torch.bool, device="cuda")
    rows = torch.arange(t, device="cuda")
    for _ in range(k):
        top = left.max(1, keepdim=True).values
        first = torch.where((left == top) & (top > -math.inf), torch.arange(e, device="cuda"), e).min(1).values
        ok = first < e
        chosen[rows[ok], first[ok]] = True
        left[rows[ok], first[ok]] = -math.inf
    z = torch.exp(l - l.max(1, keepdim=True).values).nan_to_num(0.0)
    p = (z / (z * chosen if s["normalise"] else z).sum(1, keepdim=True)).nan_to_num(0.0)
    w = torch.zeros(t * k, dtype=torch.float64, device="cuda")
    wt = torch.zeros_like(w)
    n = int(chosen.sum())
    w[:n] = p[chosen]
    wt[:n] = p.t()[chosen.t()]
    whole = (None, None, w, None, None, None, wt)
    if not s["backward"]:
        return whole
    g = torch.zeros(t, e, dtype=torch.float64, device="cuda")
    g[chosen] = s["d_weight"][:n].double()
    return whole + (p * g - p * (p * g).sum(1, keepdim=True),)


def _exact_combine(s, backward):
    y, weight = s["y"].double(), s["weight"].double()
    t = s["row_ptr"].numel() - 1
    n = int(s["row_ptr"][-1])
    row = torch.searchsorted(s["row_ptr"], torch.arange(n, device="cuda"), right=True) - 1
    slot = s["slot"][:n].long()
    out = torch.zeros(t, y.shape[1], dtype=torch.float64, device="cuda").index_add_(0, row, y[slot] * weight[:n, None])
    if not backward:
        return out
    d = s["d_out"].double()[row]
    d_y = torch.zeros_like(y)
    d_y[slot] = weight[:n, None] * d
    d_weight = torch.zeros_like(weight)
    d_weight[:n] = (y[slot] * d).sum(1)
    return out, d_y, d_weight
