"""Which kernels the layer takes with weights in 8-bit integers, and with each of the result's types (no GPU here)."""
import re

import pytest

from tests.test_rows_launches import BF16, F32, FP8, INT8, PTR, dense, launched, lib, pytestmark  # noqa: F401

F16 = 2


@pytest.mark.parametrize("tokens,route_inside", [(1, True), (16, True), (17, False), (64, False)])
@pytest.mark.parametrize("rows,kind,number", [(BF16, BF16, 0), (BF16, FP8, 1), (BF16, INT8, 2), (F16, F16, 0), (F16, FP8, 1), (F16, INT8, 2)])
def test_kernels(lib, tokens, route_inside, rows, kind, number):  # noqa: F811
    scales = {FP8: (dense(4, 2, F32), dense(2, 2, F32)), INT8: (dense(8, 512, F32), dense(8, 200, F32))}.get(kind, (None, None))
    for out in (rows, F32):
        lines = launched(lib, lib.gmagnus_expert_layer(dense(tokens, 256, rows), dense(tokens, 8, F32), 2, 1, dense(512, 256, kind), scales[0],
                                                       dense(200, 256, kind), scales[1], dense(tokens, 200, out), PTR, 1 << 40, None))
        assert len(lines) == (2 if route_inside else 3) and (route_inside or "k_layer_route" in lines[0])
        t = "DF16b" if rows == BF16 else "DF16_"
        assert re.search("k_layer_upILNS0_4KindE%dE%sLi%dELb%dE" % (number, t, 1 if route_inside else 2, route_inside), lines[-2]), lines
        assert re.search("k_layer_downILNS0_4KindE%dE%s%sE" % (number, t, "f" if out == F32 else t if rows == BF16 else "[^f]*"), lines[-1]), lines
