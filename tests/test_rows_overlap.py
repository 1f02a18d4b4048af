"""Outputs that share memory with inputs, on the host: what is refused and what is not (the library's sources are built
for the host alone, as in test_rows_launches.py; nothing is launched)."""
import ctypes
import random

import pytest

from tests.test_rows_launches import BF16, F32, FP8, INT8, gm, lib, pytestmark  # noqa: F401

SIZE = {F32: 4, BF16: 2, FP8: 1, INT8: 1}
BASE = 0x100000


def desc(at, rows, cols, stride, dtype=BF16):
    return gm.DenseDesc(BASE + at, rows, cols, stride, 0, dtype)


def cells(d):
    size = SIZE[d.data_type]
    return {d.data + r * d.row_stride * size + b for r in range(d.n_rows) for b in range(d.n_cols * size)}


def same(a, b):
    return (a.data, a.data_type, a.n_rows, a.n_cols) == (b.data, b.data_type, b.n_rows, b.n_cols) and (
        a.row_stride == b.row_stride or a.n_rows == 1)


def norm(lib, x, y, residual=None, total=None, weight=None, q=None, scale=None):  # noqa: F811
    r = lambda d: None if d is None else ctypes.byref(d)  # noqa: E731
    st = lib.gmagnus_rms_norm(r(x), r(residual), r(weight), 1e-6, r(total), r(y), r(q), r(scale), None)
    return st, lib.take_log().decode()


def test_norm_against_a_list_of_bytes(lib):  # noqa: F811
    rng = random.Random(1)
    met = [0, 0, 0]
    for _ in range(20000):
        rows, n = rng.choice([1, 1, 2, 3, 5, 9]), rng.choice([1, 2, 3, 5, 8])
        # strides alike or not, rows between one another's
        s1, s2 = n + rng.choice([0, 1, n, 2 * n, 7]), n + rng.choice([0, 1, n, 2 * n, 7])
        if rng.random() < 0.4:
            s2 = s1
        x, y = desc(2 * rng.randrange(60), rows, n, s1), desc(2 * rng.randrange(60), rows, n, s2)
        if rng.random() < 0.1:
            y.data = x.data
        meet = bool(cells(x) & cells(y))
        st, log = norm(lib, x, y)
        assert st == (1 if meet and not same(x, y) else 0), (x.data, y.data, rows, n, s1, s2, log)
        met[0 if not meet else 1 if same(x, y) else 2] += 1
    assert min(met) > 200


def test_norm_every_operand(lib):  # noqa: F811
    def case(**at):
        a = dict(x=0, residual=10000, total=20000, y=30000, weight=40000, q=50000, scale=60000)
        a.update(at)
        return norm(lib, desc(a["x"], 5, 200, 200), desc(a["y"], 5, 200, 200), desc(a["residual"], 5, 200, 200), desc(a["total"], 5, 200, 200),
                    desc(a["weight"], 1, 200, 200), desc(a["q"], 5, 200, 200, FP8), desc(a["scale"], 5, 2, 2, F32))

    assert case()[0] == 0
    for at in (dict(total=10000), dict(total=0), dict(y=0), dict(y=10000), dict(total=0, y=10000), dict(residual=0), dict(x=10000, total=10000)):
        assert case(**at)[0] == 0, at
    for at, text in ((dict(total=2), "total overlaps X"), (dict(total=10400), "total overlaps residual"), (dict(y=400), "Y overlaps X"),
                     (dict(y=20000), "Y overlaps total"), (dict(total=40300), "total overlaps weight"), (dict(q=0), "Q overlaps X"),
                     (dict(q=10008), "Q overlaps residual"), (dict(q=30000), "Q overlaps Y"), (dict(scale=1996), "scale overlaps X"),
                     (dict(scale=50996), "scale overlaps Q"), (dict(y=39996), "Y overlaps weight")):
        st, log = case(**at)
        assert st == 1 and text in log, (at, log)


def test_gradients(lib):  # noqa: F811
    lib.gmagnus_gate_backward.argtypes = [ctypes.c_void_p] * 4

    def back(d_x, total=0, d_y=10000, d_total=20000):
        ds = [desc(v, 5, 200, 200) for v in (total, d_y, d_total, d_x)]
        w = desc(40000, 1, 200, 200)
        st = lib.gmagnus_rms_norm_backward(ctypes.byref(ds[0]), ctypes.byref(w), 1e-6, *(ctypes.byref(d) for d in ds[1:]), 0x1000, 0x1000, 1 << 40, None)
        return st, lib.take_log().decode()

    for at in (0, 10000, 20000, 30000, 22000):
        assert back(at)[0] == 0
    for at, text in ((2, "TOTAL"), (10400, "D_Y"), (18002, "D_TOTAL")):
        st, log = back(at)
        assert st == 1 and "D_X overlaps " + text in log

    def gate(d_h, stride=400):
        h, d, o = desc(0, 5, 400, 400), desc(10000, 5, 200, 600), desc(d_h, 5, 400, stride)
        st = lib.gmagnus_gate_backward(ctypes.byref(h), ctypes.byref(d), ctypes.byref(o), None)
        return st, lib.take_log().decode()

    assert gate(0)[0] == 0 and gate(20000)[0] == 0 and gate(10400, 600)[0] == 0  # (the last: beside the gradient's columns)
    for at, stride, text in ((2, 400, "H"), (0, 500, "H"), (10000, 600, "D_A"), (10400 - 2, 600, "D_A")):
        st, log = gate(at, stride)
        assert st == 1 and "D_H overlaps " + text in log, log


def test_many_rows_between_one_anothers_take_no_time(lib):  # noqa: F811
    import time

    rows = (1 << 31) - 2
    t = time.perf_counter()
    assert norm(lib, desc(0, rows, 8, 16), desc(16, rows, 8, 16))[0] == 0 and norm(lib, desc(0, rows, 8, 16), desc(14, rows, 8, 16))[0] == 1
    assert time.perf_counter() - t < 0.5
