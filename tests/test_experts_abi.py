"""Argument checks of the routed expert products: every refusal is a status
code with a message and happens before a device is touched (no GPU here)."""
import ctypes
import os

import pytest
import torch

gm = pytest.importorskip("paper_2607_22866_amd.gmagnus")

F32, BF16, F16, FP8 = 0, 1, 2, 3
INVALID, UNSUPPORTED = 1, 6
PTR = 0x1000  # never read: every call below is refused


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gm.LIB_PATH):
        from paper_2607_22866_amd import build

        build.build()
    return gm.load()


def dense(n, k, dtype=BF16, ptr=PTR, stride=None, stack=None):
    return gm.DenseDesc(ptr, n, k, k if stride is None else stride, n * k if stack is None else stack, dtype)


def groups(n_groups=2, n_rows=8, gp=PTR, index=PTR):
    return gm.GroupsDesc(n_groups, n_rows, gp, index)


def routing(**kw):
    r = gm.RoutingDesc(*[PTR] * 7)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def ref(x):
    return None if x is None else ctypes.byref(x)


ROUTE_BAD = [
    (INVALID, dict(logits=None)), (INVALID, dict(out=None)), (INVALID, dict(top_k=0)), (INVALID, dict(top_k=9)),
    (INVALID, dict(normalise=2)), (INVALID, dict(logits=dense(4, 8, FP8))), (INVALID, dict(logits=dense(4, 8, 7))),
    (INVALID, dict(logits=dense(4, 8, F32, ptr=None))), (INVALID, dict(logits=dense(4, 8, F32, stride=7))),
    (INVALID, dict(logits=dense(4, 8, F32, ptr=0x1002))), (UNSUPPORTED, dict(logits=dense(4, 1025, F32))),
    (UNSUPPORTED, dict(logits=dense(1 << 30, 8, F32))), (INVALID, dict(bytes=16)), (INVALID, dict(ws=None)),
    (INVALID, dict(ws=0x1008)), (INVALID, dict(out=routing(row_ptr=None))), (INVALID, dict(out=routing(slot=None))),
]


@pytest.mark.parametrize("status,kw", ROUTE_BAD)
def test_route_refusals(lib, status, kw):
    a = dict(logits=dense(4, 8, F32), top_k=2, normalise=1, out=routing(), ws=PTR, bytes=1 << 20)
    a.update(kw)
    st = lib.gmagnus_route(ref(a["logits"]), a["top_k"], a["normalise"], ref(a["out"]), a["ws"], a["bytes"], None)
    assert st == status and lib.gmagnus_last_error()


def test_route_workspace_bytes(lib):
    f = lib.gmagnus_route_workspace_bytes
    assert f(1, 64, 4) > 0 and f(1 << 20, 256, 8) > f(1 << 10, 256, 8)
    for bad in ((4, 8, 9), (4, 8, 0), (4, 0, 1), (-1, 8, 1), (4, 1025, 1), (1 << 30, 8, 2)):
        assert f(*bad) == 0


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(d_logits=None)), (INVALID, dict(d_logits=dense(4, 8, BF16))), (INVALID, dict(d_logits=dense(4, 9, F32))),
    (INVALID, dict(d_weight=None)), (INVALID, dict(r=routing(weight=None))), (INVALID, dict(r=None))])
def test_route_backward_refusals(lib, status, kw):
    a = dict(r=routing(), d_weight=PTR, d_logits=dense(4, 8, F32))
    a.update(kw)
    assert lib.gmagnus_route_backward(ref(dense(4, 8, F32)), 2, 1, ref(a["r"]), a["d_weight"], ref(a["d_logits"]),
                                      None) == status


PRODUCT_BAD = [
    (INVALID, dict(g=None)), (INVALID, dict(x=None)), (INVALID, dict(w=None)), (INVALID, dict(y=None)),
    (INVALID, dict(g=groups(n_groups=0))), (INVALID, dict(g=groups(gp=None))), (INVALID, dict(g=groups(n_rows=-1))),
    (INVALID, dict(g=groups(index=None))),                    # X then needs n_rows rows
    (INVALID, dict(x=dense(5, 16, F32))), (INVALID, dict(x=dense(5, 16, FP8))), (INVALID, dict(x=dense(5, 16, F16))),
    (INVALID, dict(w=dense(24, 17))), (INVALID, dict(w=dense(25, 16))), (INVALID, dict(y=dense(8, 24, F16))),
    (INVALID, dict(y=dense(7, 24))), (INVALID, dict(x=dense(5, 16, stride=15))), (INVALID, dict(x=dense(5, 16, ptr=0x1001))),
    (INVALID, dict(x=dense(5, 0))), (INVALID, dict(transposed=2)), (INVALID, dict(transposed=1)),
    (INVALID, dict(w=dense(24, 16, stack=-1))),
    (UNSUPPORTED, dict(g=groups(n_rows=(1 << 31) - 1), y=dense((1 << 31) - 1, 24))),
    (UNSUPPORTED, dict(x=dense((1 << 31) - 1, 16))),
]


@pytest.mark.parametrize("status,kw", PRODUCT_BAD)
def test_group_product_refusals(lib, status, kw):
    a = dict(g=groups(), x=dense(5, 16), w=dense(24, 16), y=dense(8, 24), transposed=0)
    a.update(kw)
    st = lib.gmagnus_group_product(ref(a["g"]), ref(a["x"]), ref(a["w"]), a["transposed"], ref(a["y"]), None)
    assert st == status and lib.gmagnus_last_error()


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(dy=None)), (INVALID, dict(d=None)), (INVALID, dict(dy=dense(7, 24))), (INVALID, dict(d=dense(24, 17))),
    (INVALID, dict(dy=dense(8, 24, F16))), (INVALID, dict(d=dense(24, 16, F16))), (INVALID, dict(d=dense(24, 16, stack=383))),
    (INVALID, dict(x=dense(5, 16, F32), dy=dense(8, 24, F32)))])
def test_group_outer_refusals(lib, status, kw):
    a = dict(g=groups(), dy=dense(8, 24), x=dense(5, 16), d=dense(24, 16))
    a.update(kw)
    assert lib.gmagnus_group_outer(ref(a["g"]), ref(a["dy"]), ref(a["x"]), ref(a["d"]), None) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(x=None)), (INVALID, dict(rows=2)), (INVALID, dict(q=dense(5, 200, BF16))), (INVALID, dict(q=dense(5, 199, FP8))),
    (INVALID, dict(scale=dense(5, 3, F32))), (INVALID, dict(scale=dense(5, 2, BF16))), (INVALID, dict(x=dense(5, 200, FP8))),
    (INVALID, dict(rows=128)), (INVALID, dict(stack=-1))])
def test_quantise_refusals(lib, status, kw):
    a = dict(x=dense(5, 200), rows=1, stack=1, q=dense(5, 200, FP8), scale=dense(5, 2, F32))
    a.update(kw)
    assert lib.gmagnus_quantise_blocks(ref(a["x"]), a["stack"], a["rows"], ref(a["q"]), ref(a["scale"]), None) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(xs=None)), (INVALID, dict(x=dense(5, 200))), (INVALID, dict(xs=dense(5, 1, F32))), (INVALID, dict(xs=dense(4, 2, F32))),
    (INVALID, dict(ws=dense(2, 2, F32))), (INVALID, dict(w=dense(24, 200, BF16))), (INVALID, dict(y=dense(8, 24, FP8))),
    (INVALID, dict(ws=dense(1, 2, F16)))])
def test_fp8_refusals(lib, status, kw):
    a = dict(g=groups(), x=dense(5, 200, FP8), xs=dense(5, 2, F32), w=dense(24, 200, FP8), ws=dense(1, 2, F32), y=dense(8, 24))
    a.update(kw)
    assert lib.gmagnus_group_product_fp8(ref(a["g"]), ref(a["x"]), ref(a["xs"]), ref(a["w"]), ref(a["ws"]), ref(a["y"]),
                                         None) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(rp=None)), (INVALID, dict(slot=None)), (INVALID, dict(y=None)), (INVALID, dict(out=None)),
    (INVALID, dict(y=dense(8, 25))), (INVALID, dict(y=dense(8, 24, F16))), (INVALID, dict(out=dense(4, 24, FP8), y=dense(8, 24, FP8))),
    (INVALID, dict(n=-1)), (UNSUPPORTED, dict(n=1 << 31)), (INVALID, dict(out=dense(4, 0), y=dense(8, 0)))])
def test_combine_refusals(lib, status, kw):
    a = dict(rp=PTR, slot=PTR, n=8, y=dense(8, 24), out=dense(4, 24))
    a.update(kw)
    assert lib.gmagnus_combine(a["rp"], a["slot"], None, a["n"], ref(a["y"]), ref(a["out"]), None) == status
    # the gradients: the sum's gradient takes OUT's place
    assert lib.gmagnus_combine_backward(a["rp"], a["slot"], None, a["n"], ref(a["y"]), ref(a["out"]), ref(dense(8, 24)), PTR,
                                        None) == status


def test_combine_backward_wants_something(lib):
    assert lib.gmagnus_combine_backward(PTR, PTR, None, 8, ref(dense(8, 24)), ref(dense(4, 24)), None, None, None) == INVALID
    assert lib.gmagnus_combine_backward(PTR, PTR, None, 8, ref(dense(8, 24)), ref(dense(4, 24)), ref(dense(9, 24)), PTR,
                                        None) == INVALID


def test_binding_refuses_host_tensors(lib):
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, 6, 8, dtype=torch.bfloat16)
    gp = torch.zeros(3, dtype=torch.int64)
    for call in (lambda: gm.route(x, 2), lambda: gm.group_product(x, w, gp), lambda: gm.group_outer(x, x, gp),
                 lambda: gm.quantise_blocks(x), lambda: gm.combine(x, gp, gp.int()),
                 lambda: gm.combine_backward(x, gp, gp.int(), None, x)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()


@pytest.mark.parametrize("stride", [0, -24, 23])
def test_single_rows_need_their_stride(lib, stride):
    # (a gradient's rows are the reduction: rows past the last are told apart by the stride, also past a single one)
    g, x, d = groups(n_rows=1), dense(1, 16), dense(24, 16)
    assert lib.gmagnus_group_outer(ref(g), ref(dense(1, 24, stride=stride)), ref(x), ref(d), None) == INVALID
    assert b"row stride" in lib.gmagnus_last_error()


@pytest.mark.parametrize("kw", [dict(q=dense(5, 200, FP8, stack=999)), dict(q=dense(5, 200, FP8, stride=208, stack=1031)),
                                dict(scale=dense(5, 2, F32, stack=0))])
def test_quantised_stacks_do_not_overlap(lib, kw):
    a = dict(q=dense(5, 200, FP8), scale=dense(5, 2, F32))
    a.update(kw)
    assert lib.gmagnus_quantise_blocks(ref(dense(5, 200)), 3, 1, ref(a["q"]), ref(a["scale"]), None) == INVALID
    assert b"overlap" in lib.gmagnus_last_error()
