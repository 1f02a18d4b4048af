"""Which kernels the calls around the products take (no GPU here): the library's sources are built for the host alone
and linked with stubs that write launches down, as test_experts_launches.py does it."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from tests import int8_cases as ic

gm = pytest.importorskip("paper_2607_22866_amd.gmagnus")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_22866_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
F32, BF16, FP8, INT8 = 0, 1, 3, 4
PTR = 0x1000  # never read: nothing is launched

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC) or shutil.which("g++") is None, reason="needs hipcc and g++")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("rows_launches")

    def run(*cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
        return r.stdout

    objs = [str(tmp / "stubs.o")]
    run("g++", "-O1", "-fPIC", "-std=c++17", "-c", os.path.join(ROOT, "tests", "launches", "stubs.cpp"), "-o", objs[0])
    for f in ("group_int8", "rows", "layer"):
        objs.append(str(tmp / (f + ".o")))
        run(HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-std=c++17", "-I",
            os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, f + ".hip"), "-o", objs[-1])
    device = sorted(set(re.findall(r"__hip_fatbin_\w+", run("nm", "-u", *objs))))
    so = str(tmp / "liblaunches.so")
    run("g++", "-shared", "-o", so, *objs, *["-Wl,--defsym=%s=0" % d for d in device])
    lib = ctypes.CDLL(so)
    lib.take_log.restype = ctypes.c_char_p
    lib.gmagnus_rms_norm.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_double] + [ctypes.c_void_p] * 5
    lib.gmagnus_rms_norm_backward.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_double] + [ctypes.c_void_p] * 5 + [ctypes.c_int64, ctypes.c_void_p]
    lib.gmagnus_expert_layer.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int64, ctypes.c_int32] + [ctypes.c_void_p] * 6 + [ctypes.c_int64, ctypes.c_void_p]
    return lib


def dense(n, k, dtype=BF16):
    return ctypes.byref(gm.DenseDesc(PTR, n, k, k, n * k, dtype))


def launched(lib, status):
    log = lib.take_log().decode()
    assert status == 0, log
    lines = log.splitlines()
    assert all(line.startswith("launch ") for line in lines), log
    return lines


@pytest.mark.parametrize("kernel,sizes,n,k", ic.PRODUCTS)
def test_integer_products(lib, kernel, sizes, n, k):
    rows, groups = sum(sizes), len(sizes)
    g = ctypes.byref(gm.GroupsDesc(groups, rows, PTR, PTR))
    for out in (BF16, F32):
        line, = launched(lib, lib.gmagnus_group_product_int8(g, dense(rows, k, INT8), dense(1, rows, F32), dense(n, k, INT8),
                                                             dense(groups, n, F32), dense(rows, n, out), None))
        assert re.search(ic.KERNELS[kernel], line), line


def test_every_integer_kernel_has_a_case():
    assert {c[0] for c in ic.PRODUCTS} == set(ic.KERNELS)


@pytest.mark.parametrize("n,waves,pieces", [(1, 1, 1), (512, 1, 1), (513, 1, 2), (1024, 1, 2), (1025, 4, 1), (2048, 4, 1), (2049, 4, 2),
                                            (4096, 4, 2), (4097, 8, 2), (8192, 8, 2), (8193, 16, 2), (16384, 16, 2), (16385, 0, 0)])
def test_rows(lib, n, waves, pieces):
    whole = "Lb%d" % (n % 8 == 0)
    name = "k_rows.*Li%dELi%dE%sE" % (waves, pieces, whole) if waves else "k_rows_long.*%sE" % whole
    line, = launched(lib, lib.gmagnus_rms_norm(dense(9000, n), None, None, 1e-6, None, dense(9000, n), None, None, None))
    assert re.search(name, line), line
    line, = launched(lib, lib.gmagnus_gate(dense(9, 2 * n), dense(9, n), None, None, None))
    assert re.search(name, line), line
    lines = launched(lib, lib.gmagnus_rms_norm_backward(dense(9000, n), dense(1, n), 1e-6, dense(9000, n), None, dense(9000, n), PTR, PTR,
                                                        1 << 40, None))
    if n <= 8192:
        assert len(lines) == 2 and re.search("k_norm_backwardI.*Li%dELi%dE%sE" % (waves, pieces, whole), lines[0]), lines
    else:
        assert len(lines) == 3 and "k_norm_backward_rows" in lines[0] and "k_norm_backward_columns" in lines[1], lines
    assert "k_add_shares" in lines[-1]


@pytest.mark.parametrize("tokens,kernels", [(1, 2), (16, 2), (17, 3), (64, 3)])
@pytest.mark.parametrize("fp8", [False, True])
def test_layer(lib, tokens, kernels, fp8):
    kind = FP8 if fp8 else BF16
    s1, s2 = (dense(4, 2, F32), dense(2, 2, F32)) if fp8 else (None, None)
    lines = launched(lib, lib.gmagnus_expert_layer(dense(tokens, 256), dense(tokens, 8, F32), 2, 1, dense(512, 256, kind), s1,
                                                   dense(200, 256, kind), s2, dense(tokens, 200), PTR, 1 << 40, None))
    assert len(lines) == kernels and "k_layer_up" in lines[-2] and "k_layer_down" in lines[-1], lines
    assert kernels == 2 or "k_layer_route" in lines[0]
