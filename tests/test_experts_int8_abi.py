"""Argument checks of the products of 8-bit integers: every refusal is a status code with a message and happens before
a device is touched (no GPU here)."""
import pytest

from tests.test_experts_abi import BF16, F16, F32, FP8, INVALID, PTR, UNSUPPORTED, dense, gm, groups, lib, ref  # noqa: F401

INT8 = 4


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(g=None)), (INVALID, dict(x=None)), (INVALID, dict(xs=None)), (INVALID, dict(w=None)), (INVALID, dict(ws=None)),
    (INVALID, dict(y=None)), (INVALID, dict(x=dense(5, 200))), (INVALID, dict(x=dense(5, 200, FP8))), (INVALID, dict(xs=dense(5, 1, F32))),
    (INVALID, dict(xs=dense(1, 4, F32))), (INVALID, dict(xs=dense(1, 5, F16))), (INVALID, dict(w=dense(24, 200, FP8))),
    (INVALID, dict(w=dense(24, 199, INT8))), (INVALID, dict(ws=dense(1, 24, F32))), (INVALID, dict(ws=dense(2, 23, F32))),
    (INVALID, dict(ws=dense(2, 24, F32, stride=23))), (INVALID, dict(ws=dense(2, 24, BF16))), (INVALID, dict(y=dense(8, 24, FP8))),
    (INVALID, dict(y=dense(8, 24, INT8))), (INVALID, dict(y=dense(7, 24))), (INVALID, dict(g=groups(index=None))),
    (INVALID, dict(w=dense(24, 200, INT8, stack=-1))), (INVALID, dict(x=dense(5, 200, INT8, stride=199))),
    (UNSUPPORTED, dict(x=dense(5, 131072, INT8), w=dense(24, 131072, INT8))), (UNSUPPORTED, dict(g=groups(n_rows=(1 << 31) - 1)))])
def test_refusals(lib, status, kw):  # noqa: F811
    a = dict(g=groups(), x=dense(5, 200, INT8), xs=dense(1, 5, F32), w=dense(24, 200, INT8), ws=dense(2, 24, F32), y=dense(8, 24))
    a.update(kw)
    st = lib.gmagnus_group_product_int8(ref(a["g"]), ref(a["x"]), ref(a["xs"]), ref(a["w"]), ref(a["ws"]), ref(a["y"]), None)
    assert st == status and lib.gmagnus_last_error()
