"""Every load from memory straight into LDS is checked against its operand's
end as a whole: its scalar offset is 0, so the lane's offset, which is compared
with the operand's bytes, says all of where it reads. (A scalar offset is not
compared as the lane's offset is: the tiles' steps past the last one read up to 8
bytes past the scales' last row through it.) Checked on the disassembly of the
built library."""
import os
import re

import pytest

from paper_2607_22866_amd.build import LIB
from tests.test_barrier_waits import OBJDUMP, _kernels

LOAD = re.compile(r"buffer_load_\w+ \S+ s\[\d+:\d+\], (\S+)(.*) lds\b")


def scalar_offsets(body):
    """The scalar offsets of a function's buffer loads into LDS."""
    return [m.group(1) for m in (LOAD.match(s) for _, s in body) if m]


def test_parser_sees_offsets():
    body = [(0, "buffer_load_dwordx4 v1, s[4:7], s9 offen lds"), (8, "buffer_load_dword v1, s[4:7], 0 offen lds"),
            (16, "buffer_load_dwordx4 v[0:3], v1, s[4:7], s9 offen")]
    assert scalar_offsets(body) == ["s9", "0"]


def test_loads_into_lds_have_no_scalar_offset(tmp_path):
    if not (os.path.exists(OBJDUMP) and os.path.exists(LIB)):
        pytest.skip("needs llvm-objdump and the built library")
    loads, bad = 0, {}
    for name, body in _kernels(tmp_path):
        found = scalar_offsets(body)
        loads += len(found)
        if any(o != "0" for o in found):
            bad[name] = sorted(set(found))
    assert loads > 100
    assert not bad, bad
