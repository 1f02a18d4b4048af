"""The largest calls around the products stay below the 2^32 threads that a launch may have (no GPU here)."""
import ctypes
import re

import pytest

from tests.test_rows_launches import BF16, F32, INT8, PTR, dense, gm, launched, lib, pytestmark  # noqa: F401

LIMIT = 1 << 32
UNSUPPORTED = 6


def threads(line):
    """Of a launch: its work groups times the kernel's largest (what its name says of the waves, at least 256)."""
    m = re.search(r"k_rowsI.*Li(\d+)ELi\d+ELb", line) or re.search(r"k_norm_backwardI.*Li(\d+)ELi\d+ELb", line)
    wave = {"k_rows_long": 1024, "k_add_shares": 1024, "k_norm_backward_rows": 1024, "k_norm_backward_columns": 64}
    per = next((v for k, v in wave.items() if k in line), max(256, 64 * int(m.group(1))) if m else 256)
    return int(line.split()[2]) * per


@pytest.mark.parametrize("n", [8, 1000, 2048, 4096, 8192, 9000, 16384, 20000])
@pytest.mark.parametrize("rows", [1, 1 << 20, (1 << 22) + 5, (1 << 31) - 2])
def test_rows(lib, rows, n):  # noqa: F811
    y, q = dense(rows, n), dense(rows, n, INT8)
    lib.gmagnus_quantise_rows.argtypes = [ctypes.c_void_p, ctypes.c_int64] + [ctypes.c_void_p] * 3
    lib.gmagnus_gate_backward.argtypes = [ctypes.c_void_p] * 4
    far = gm.DenseDesc(1 << 60, rows, n, n, 0, BF16)
    for status in (lib.gmagnus_rms_norm(y, None, None, 1e-6, None, y, None, None, None), lib.gmagnus_gate(dense(rows, 2 * n), y, None, None, None),
                   lib.gmagnus_quantise_rows(y, 1, q, dense(1, rows, F32), None),
                   lib.gmagnus_gate_backward(dense(rows, 2 * n), ctypes.byref(far), dense(rows, 2 * n), None),
                   lib.gmagnus_rms_norm_backward(y, dense(1, n), 1e-6, y, None, y, PTR, PTR, 1 << 60, None)):
        for line in launched(lib, status):
            assert threads(line) < LIMIT, line


@pytest.mark.parametrize("n", [(1 << 28) - 64, 1 << 28, (1 << 31) - 1032])
def test_one_long_row(lib, n):  # noqa: F811
    x = dense(1, n)
    for line in launched(lib, lib.gmagnus_rms_norm_backward(x, x, 1e-6, x, None, x, PTR, PTR, 1 << 60, None)):
        assert threads(line) < LIMIT, line


def test_columns_of_the_layer(lib):  # noqa: F811
    def layer(n):
        return lib.gmagnus_expert_layer(dense(1, 64), dense(1, 2, F32), 1, 1, dense(64, 64), None, dense(n, 32), None, dense(1, n), PTR, 1 << 60, None)

    lines = launched(lib, layer((1 << 29) - 32))
    assert int(lines[-1].split()[2]) == (1 << 24) - 1 and threads(lines[-1]) < LIMIT
    lib.gmagnus_expert_layer_workspace_bytes.restype = ctypes.c_int64
    f = lambda n: lib.gmagnus_expert_layer_workspace_bytes(*(ctypes.c_int64(v) for v in (1, 2, 1, 32, n)))  # noqa: E731
    assert f((1 << 29) - 32) > 0 and f((1 << 29) - 31) == 0
    assert layer((1 << 29) - 31) == UNSUPPORTED and "beyond 2^29 - 32" in lib.take_log().decode()
