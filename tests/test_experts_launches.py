"""Which kernel the grouped products take (no GPU here): the library's sources are
built for the host alone and linked with stubs that write launches down. The
cases of experts_cases.py, which the GPU tests run, reach the kernels they name:
both sides of every limit, and every kernel's inner loops."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from tests import experts_cases as ec

gm = pytest.importorskip("paper_2607_22866_amd.gmagnus")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_22866_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
BF16, F32, FP8 = 1, 0, 3
PTR = 0x1000  # never read: nothing is launched

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC) or shutil.which("g++") is None, reason="needs hipcc and g++")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("launches")

    def run(*cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
        return r.stdout

    objs = [str(tmp / "stubs.o")]
    run("g++", "-O1", "-fPIC", "-std=c++17", "-c", os.path.join(ROOT, "tests", "launches", "stubs.cpp"), "-o", objs[0])
    for f in ("group", "group_fp8"):
        objs.append(str(tmp / (f + ".o")))
        run(HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-fPIC", "-std=c++17", "-I",
            os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, f + ".hip"), "-o", objs[-1])
    # (device code is not there: its symbols stand for nothing)
    device = sorted(set(re.findall(r"__hip_fatbin_\w+", run("nm", "-u", *objs))))
    so = str(tmp / "liblaunches.so")
    run("g++", "-shared", "-o", so, *objs, *["-Wl,--defsym=%s=0" % d for d in device])
    lib = ctypes.CDLL(so)
    lib.take_log.restype = ctypes.c_char_p
    return lib


def dense(n, k, dtype=BF16):
    return ctypes.byref(gm.DenseDesc(PTR, n, k, k, n * k, dtype))


def launched(lib, status):
    log = lib.take_log().decode()
    assert status == 0, log
    lines = log.splitlines()
    assert len(lines) == 1 and lines[0].startswith("launch "), log
    return lines[0]


def check(line, kernel):
    assert re.search(ec.KERNELS[kernel], line), line


@pytest.mark.parametrize("kernel,sizes,n,k,transposed", ec.PRODUCTS)
def test_products(lib, kernel, sizes, n, k, transposed):
    rows = sum(sizes)
    g = gm.GroupsDesc(len(sizes), rows, PTR, PTR)
    w = dense(k, n) if transposed else dense(n, k)
    for out in (BF16, F32):
        check(launched(lib, lib.gmagnus_group_product(ctypes.byref(g), dense(rows, k), w, int(transposed), dense(rows, n, out), None)),
              kernel)


@pytest.mark.parametrize("kernel,sizes,n,k", ec.FP8_PRODUCTS)
def test_fp8_products(lib, kernel, sizes, n, k):
    rows, kb = sum(sizes), -(-k // 128)
    g = gm.GroupsDesc(len(sizes), rows, PTR, PTR)
    check(launched(lib, lib.gmagnus_group_product_fp8(ctypes.byref(g), dense(rows, k, FP8), dense(rows, kb, F32), dense(n, k, FP8),
                                                      dense(-(-n // 128), kb, F32), dense(rows, n), None)), kernel)


@pytest.mark.parametrize("kernel,by_size,sizes,n,k", ec.OUTERS)
def test_outers(lib, kernel, by_size, sizes, n, k):
    rows = sum(sizes)
    g = gm.GroupsDesc(len(sizes), rows, PTR, PTR)
    line = launched(lib, lib.gmagnus_group_outer(ctypes.byref(g), dense(rows, n), dense(rows, k), dense(n, k), None))
    check(line, kernel)
    assert line.endswith("by_size") == by_size, line


def test_every_kernel_has_a_case():
    used = {c[0] for c in ec.PRODUCTS + ec.FP8_PRODUCTS + ec.OUTERS}
    assert used == set(ec.KERNELS)


def test_aligned_operands_leave_the_fast_tiles_where_offsets_pass_31_bits(lib):
    # an indexed X of 2 GiB, and one just below
    for rows, kernel in (((1 << 19) - 2, "t256"), (1 << 19, "any")):
        g = gm.GroupsDesc(16, 8192, PTR, PTR)
        check(launched(lib, lib.gmagnus_group_product(ctypes.byref(g), dense(rows, 2048), dense(2048, 2048), 0, dense(8192, 2048), None)),
              kernel)
        g = gm.GroupsDesc(16, rows, PTR, None)  # (without an index each tile has offsets of its own)
        check(launched(lib, lib.gmagnus_group_product(ctypes.byref(g), dense(rows, 2048), dense(2048, 2048), 0, dense(rows, 2048), None)),
              "t256")
