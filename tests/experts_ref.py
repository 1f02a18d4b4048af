"""64-bit forms of the routed expert products on the host (numpy), for the tests."""
import numpy as np

BLOCK = 128
U = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}  # rounding to nearest, relative
TINY = {"bfloat16": 2.0 ** -133, "float16": 2.0 ** -24, "float32": 2.0 ** -149}  # and for subnormal results


def route(logits, top_k, normalise):
    """logits: float64 [T, E]. Returns a dict of the routing's arrays (weights float64)."""
    t, e = logits.shape
    l = np.where(np.isnan(logits), -np.inf, logits)
    row_ptr, expert, weight, prob = [0], [], [], np.zeros((t, e))
    for i in range(t):
        order = sorted((j for j in range(e) if l[i, j] > -np.inf), key=lambda j: (-l[i, j], j))
        chosen = sorted(order[:top_k])
        if order:
            with np.errstate(invalid="ignore"):
                z = np.where(l[i] > -np.inf, np.exp(l[i] - l[i].max()), 0.0)
            prob[i] = z / (z[chosen].sum() if normalise else z.sum())
        expert += chosen
        weight += [prob[i, j] for j in chosen]
        row_ptr.append(len(expert))
    n = len(expert)
    token = np.repeat(np.arange(t), np.diff(row_ptr))
    order = np.lexsort((token, expert))
    slot = np.empty(n, dtype=np.int64)
    slot[order] = np.arange(n)
    group_ptr = np.concatenate([[0], np.cumsum(np.bincount(np.array(expert, dtype=np.int64), minlength=e))])

    def whole(v, empty, dtype):
        out = np.full(t * top_k, empty, dtype=dtype)
        out[:n] = v
        return out

    w = np.array(weight, dtype=np.float64)
    return {"row_ptr": np.array(row_ptr), "expert": whole(expert, -1, np.int64), "weight": whole(w, 0.0, np.float64),
            "group_ptr": group_ptr, "token": whole(token[order], -1, np.int64), "slot": whole(slot, -1, np.int64),
            "group_weight": whole(w[order], 0.0, np.float64), "prob": prob, "n": n}


def route_loss(logits, d_weight, ref, normalise):
    """sum of d_weight * weight for the choice in ref, as a function of the logits."""
    total = 0.0
    for i in range(logits.shape[0]):
        b, f = ref["row_ptr"][i], ref["row_ptr"][i + 1]
        if f > b:
            ids = ref["expert"][b:f]
            z = np.exp(logits[i] - logits[i].max())
            total += float(np.dot(d_weight[b:f], z[ids] / (z[ids].sum() if normalise else z.sum())))
    return total


def rows_of(x, index, begin, end):
    """x[index[begin:end]], a row of zeros where the index names none."""
    ids = np.arange(begin, end) if index is None else index[begin:end]
    out = np.zeros((end - begin, x.shape[1]))
    ok = (ids >= 0) & (ids < x.shape[0])
    out[ok] = x[ids[ok]]
    return out


def group_product(x, w, gp, index, n_rows, transposed):
    """(values, sums of magnitudes), float64 [n_rows, N]."""
    n = w.shape[2] if transposed else w.shape[1]
    y, mag = np.zeros((n_rows, n)), np.zeros((n_rows, n))
    for e in range(len(gp) - 1):
        b, f = int(gp[e]), int(gp[e + 1])
        m = w[e] if transposed else w[e].T
        rows = rows_of(x, index, b, f)
        y[b:f] = rows @ m
        mag[b:f] = np.abs(rows) @ np.abs(m)
    return y, mag


def group_outer(d_y, x, gp, index):
    e = len(gp) - 1
    d = np.zeros((e, d_y.shape[1], x.shape[1]))
    mag = np.zeros_like(d)
    for i in range(e):
        b, f = int(gp[i]), int(gp[i + 1])
        rows = rows_of(x, index, b, f)
        d[i] = d_y[b:f].T @ rows
        mag[i] = np.abs(d_y[b:f]).T @ np.abs(rows)
    return d, mag


def bound(y, mag, terms, dtype, slack=2.0 ** -23):
    """Rounding of the result plus fp32 sums of `terms` products (each addition off by at most 2^-23 of the magnitudes)."""
    return U[dtype] * np.abs(y) + TINY[dtype] + (terms + 8) * slack * mag


def spread_scale(scale, rows, n, k):
    """A scale for each value."""
    return np.repeat(np.repeat(scale, rows, axis=-2), BLOCK, axis=-1)[..., :n, :k]
