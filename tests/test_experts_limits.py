"""Sizes at the ends of what the routed expert products accept: refused with a
status before a device is touched (no GPU here). A kernel's 32-bit counters go
past a reduction's or a group's end by up to 384 elements before they are
compared, so sizes within 1024 of 2^31 would wrap: reads at negative offsets, loops that
need not end, results left unwritten."""
import ctypes
import os

import pytest

gm = pytest.importorskip("paper_2607_22866_amd.gmagnus")

BF16, F32, FP8 = 1, 0, 3
UNSUPPORTED = 6
PTR = 0x1000  # never read: every call below is refused
SIZES = [(1 << 31) - 1024, (1 << 31) - 130, (1 << 31) - 2]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gm.LIB_PATH):
        from paper_2607_22866_amd import build

        build.build()
    return gm.load()


def dense(n, k, dtype=BF16):
    return ctypes.byref(gm.DenseDesc(PTR, n, k, k, n * k, dtype))


def groups(n_rows, index=PTR):
    return ctypes.byref(gm.GroupsDesc(1, n_rows, PTR, index))


@pytest.mark.parametrize("size", SIZES)
def test_product_sizes(lib, size):
    for tr in (0, 1):
        # a long reduction, wide results, many rows
        assert lib.gmagnus_group_product(groups(1), dense(1, size), dense(*((size, 1) if tr else (1, size))), tr, dense(1, 1),
                                         None) == UNSUPPORTED
        assert lib.gmagnus_group_product(groups(1), dense(1, 1), dense(*((1, size) if tr else (size, 1))), tr,
                                         dense(1, size), None) == UNSUPPORTED
        assert lib.gmagnus_group_product(groups(size, None), dense(size, 1), dense(1, 1), tr, dense(size, 1),
                                         None) == UNSUPPORTED
    assert b"2^31" in lib.gmagnus_last_error()


@pytest.mark.parametrize("size", SIZES)
def test_outer_sizes(lib, size):
    assert lib.gmagnus_group_outer(groups(size, None), dense(size, 1), dense(size, 1), dense(1, 1), None) == UNSUPPORTED
    assert lib.gmagnus_group_outer(groups(1), dense(1, size), dense(1, 1), dense(size, 1), None) == UNSUPPORTED
    assert lib.gmagnus_group_outer(groups(1), dense(1, 1), dense(1, size), dense(1, size), None) == UNSUPPORTED


@pytest.mark.parametrize("size", SIZES)
def test_fp8_sizes(lib, size):
    kb = -(-size // 128)
    assert lib.gmagnus_group_product_fp8(groups(1), dense(1, size, FP8), dense(1, kb, F32), dense(1, size, FP8),
                                         dense(1, kb, F32), dense(1, 1), None) == UNSUPPORTED
    assert lib.gmagnus_group_product_fp8(groups(size, None), dense(size, 1, FP8), dense(size, 1, F32), dense(1, 1, FP8),
                                         dense(1, 1, F32), dense(size, 1), None) == UNSUPPORTED
    assert lib.gmagnus_quantise_blocks(dense(1, size), 1, 1, dense(1, size, FP8), dense(1, kb, F32), None) == UNSUPPORTED
