"""A kernel's dynamic LDS begins behind its static LDS. Kernels that keep 16-byte values in the former (the layer's
sums, the tiles brought from memory) have a static part of whole 16 bytes, or those values would lie across what the
compiler takes their alignment for. Checked on the kernels' descriptions in the built library."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_22866_amd.build import LIB
from tests.test_barrier_waits import OBJDUMP

READELF = os.path.join(os.path.dirname(OBJDUMP), "llvm-readelf")
DYNAMIC = re.compile(r"k_layer_(route|up|down)|k_group_\w+_fast")


def static_lds(tmp_path):
    """(kernel, bytes of static LDS) of every kernel of the library's gfx950 code."""
    lib = shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    for f in sorted(os.listdir(tmp_path)):
        if f.endswith("gfx950"):
            notes = subprocess.run([READELF, "--notes", f], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
            for size, name in re.findall(r"\.group_segment_fixed_size: (\d+).*?\n\s+\.name:\s+(\S+)", notes, re.S):
                yield name, int(size)


def test_dynamic_lds_begins_at_16_bytes(tmp_path):
    if not (os.path.exists(OBJDUMP) and os.path.exists(READELF) and os.path.exists(LIB)):
        pytest.skip("needs llvm-objdump, llvm-readelf and the built library")
    kernels = [(n, b) for n, b in static_lds(tmp_path) if DYNAMIC.search(n)]
    assert {k for k in ("k_layer_route", "k_layer_up", "k_layer_down") if any(k in n for n, _ in kernels)} == {
        "k_layer_route", "k_layer_up", "k_layer_down"}
    assert sum("_fast" in n for n, _ in kernels) > 10
    assert [(n, b) for n, b in kernels if b % 16] == []
