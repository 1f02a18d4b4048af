"""Argument checks of the norm, the gate and the rounding of rows: every refusal is a status code with a
message and happens before a device is touched (no GPU here)."""
import pytest
import torch

from tests.test_experts_abi import BF16, F16, F32, FP8, INVALID, PTR, UNSUPPORTED, dense, gm, lib, ref  # noqa: F401

INT8 = 4
BIG = (1 << 31) - 1


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(x=None)), (INVALID, dict(x=dense(5, 0))), (INVALID, dict(x=dense(5, 200, FP8))), (INVALID, dict(x=dense(5, 200, INT8))),
    (INVALID, dict(x=dense(5, 200, stride=199))), (INVALID, dict(x=dense(5, 200, ptr=None))), (INVALID, dict(x=dense(5, 200, ptr=0x1001))),
    (INVALID, dict(total=None)), (INVALID, dict(residual=None)), (INVALID, dict(residual=dense(4, 200))), (INVALID, dict(residual=dense(5, 200, F16))),
    (INVALID, dict(total=dense(5, 200, F32))), (INVALID, dict(weight=dense(1, 199))), (INVALID, dict(weight=dense(2, 200))),
    (INVALID, dict(weight=dense(1, 200, F16))), (INVALID, dict(eps=-1e-9)), (INVALID, dict(eps=float("nan"))), (INVALID, dict(eps=float("inf"))),
    (INVALID, dict(y=None, q=None, scale=None)), (INVALID, dict(q=None)), (INVALID, dict(scale=None)), (INVALID, dict(y=dense(5, 200, F16))),
    (INVALID, dict(q=dense(5, 200, BF16))), (INVALID, dict(q=dense(5, 199, FP8))), (INVALID, dict(scale=dense(5, 1, F32))),
    (INVALID, dict(scale=dense(5, 2, BF16))), (INVALID, dict(q=dense(5, 200, INT8))),  # (its scale is 1 x 5)
    (UNSUPPORTED, dict(x=dense(BIG, 200))), (UNSUPPORTED, dict(x=dense(5, BIG - 1023))), (INVALID, dict(x=dense(-1, 200)))])
def test_rms_norm_refusals(lib, status, kw):  # noqa: F811
    a = dict(x=dense(5, 200), residual=dense(5, 200), weight=dense(1, 200), eps=1e-6, total=dense(5, 200), y=dense(5, 200),
             q=dense(5, 200, FP8), scale=dense(5, 2, F32))
    a.update(kw)
    st = lib.gmagnus_rms_norm(ref(a["x"]), ref(a["residual"]), ref(a["weight"]), a["eps"], ref(a["total"]), ref(a["y"]), ref(a["q"]),
                              ref(a["scale"]), None)
    assert st == status and lib.gmagnus_last_error()


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(h=None)), (INVALID, dict(d_y=None)), (INVALID, dict(d_x=None)), (INVALID, dict(h=dense(5, 200, FP8))),
    (INVALID, dict(d_y=dense(5, 199))), (INVALID, dict(d_y=dense(5, 200, F16))), (INVALID, dict(d_total=dense(4, 200))),
    (INVALID, dict(d_x=dense(5, 200, F32))), (INVALID, dict(weight=dense(1, 200, F16))), (INVALID, dict(eps=float("nan"))),
    (INVALID, dict(d_weight=0x1002)), (INVALID, dict(ws=None)), (INVALID, dict(ws=0x1008)), (INVALID, dict(bytes=64)),
    (UNSUPPORTED, dict(h=dense(BIG, 200)))])
def test_rms_norm_backward_refusals(lib, status, kw):  # noqa: F811
    a = dict(h=dense(5, 200), weight=dense(1, 200), eps=1e-6, d_y=dense(5, 200), d_total=None, d_x=dense(5, 200), d_weight=PTR, ws=PTR,
             bytes=1 << 20)
    a.update(kw)
    st = lib.gmagnus_rms_norm_backward(ref(a["h"]), ref(a["weight"]), a["eps"], ref(a["d_y"]), ref(a["d_total"]), ref(a["d_x"]),
                                       a["d_weight"], a["ws"], a["bytes"], None)
    assert st == status and lib.gmagnus_last_error()


def test_rms_norm_backward_workspace_bytes(lib):  # noqa: F811
    f = lib.gmagnus_rms_norm_backward_workspace_bytes
    assert f(1, 1) > 0 and f(1 << 20, 4096) >= 512 * 4096 * 4 and f(1 << 20, 40000) >= (512 * 40000 + 2 * (1 << 20)) * 4
    for bad in ((-1, 8), (8, 0), (BIG, 8), (8, BIG - 1023)):
        assert f(*bad) == 0


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(h=None)), (INVALID, dict(h=dense(5, 399))), (INVALID, dict(h=dense(5, 400, INT8))), (INVALID, dict(y=dense(5, 400))),
    (INVALID, dict(y=None)), (INVALID, dict(y=dense(5, 200, F32))), (INVALID, dict(q=dense(5, 200, INT8))),
    (INVALID, dict(q=dense(5, 200, INT8), scale=dense(5, 1, F32))), (UNSUPPORTED, dict(h=dense(BIG, 400)))])
def test_gate_refusals(lib, status, kw):  # noqa: F811
    a = dict(h=dense(5, 400), y=dense(5, 200), q=None, scale=None)
    a.update(kw)
    assert lib.gmagnus_gate(ref(a["h"]), ref(a["y"]), ref(a["q"]), ref(a["scale"]), None) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(h=None)), (INVALID, dict(d_y=None)), (INVALID, dict(d_h=None)), (INVALID, dict(h=dense(5, 401))),
    (INVALID, dict(d_y=dense(5, 400))), (INVALID, dict(d_h=dense(5, 200))), (INVALID, dict(d_h=dense(5, 400, F16)))])
def test_gate_backward_refusals(lib, status, kw):  # noqa: F811
    a = dict(h=dense(5, 400), d_y=dense(5, 200), d_h=dense(5, 400))
    a.update(kw)
    assert lib.gmagnus_gate_backward(ref(a["h"]), ref(a["d_y"]), ref(a["d_h"]), None) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(x=None)), (INVALID, dict(q=None)), (INVALID, dict(scale=None)), (INVALID, dict(x=dense(5, 200, INT8))),
    (INVALID, dict(q=dense(5, 200, FP8))), (INVALID, dict(scale=dense(5, 3, F32))), (INVALID, dict(scale=dense(3, 4, F32))),
    (INVALID, dict(scale=dense(3, 5, F16))), (INVALID, dict(stack=-1)), (INVALID, dict(q=dense(5, 200, INT8, stack=999))),
    (INVALID, dict(scale=dense(3, 5, F32, stride=4))), (UNSUPPORTED, dict(stack=1 << 31))])
def test_quantise_rows_refusals(lib, status, kw):  # noqa: F811
    a = dict(x=dense(5, 200), stack=3, q=dense(5, 200, INT8), scale=dense(3, 5, F32))
    a.update(kw)
    assert lib.gmagnus_quantise_rows(ref(a["x"]), a["stack"], ref(a["q"]), ref(a["scale"]), None) == status


def test_integers_are_refused_where_no_call_names_them(lib):  # noqa: F811
    x = dense(5, 200, INT8)
    assert lib.gmagnus_quantise_blocks(ref(x), 1, 1, ref(dense(5, 200, FP8)), ref(dense(5, 2, F32)), None) == INVALID
    assert b"unknown data type" in lib.gmagnus_last_error()
    with pytest.raises(ValueError, match="CUDA tensor"):
        gm.rms_norm(torch.zeros(4, 8))
    with pytest.raises(ValueError, match="CUDA tensor"):
        gm.gate(torch.zeros(4, 8))
