"""Argument checks of the layer of experts for a few tokens: every refusal is a status code with a message and
happens before a device is touched (no GPU here)."""
import pytest
import torch

from tests.test_experts_abi import BF16, F16, F32, FP8, INVALID, PTR, UNSUPPORTED, dense, gm, lib, ref  # noqa: F401

INT8 = 4
BIG = 1 << 30


def fp8(**kw):
    return dict(dict(w1=dense(300, 200, FP8), s1=dense(3, 2, F32), w2=dense(96, 150, FP8), s2=dense(1, 2, F32)), **kw)


def int8(**kw):
    return dict(dict(w1=dense(300, 200, INT8), s1=dense(8, 300, F32), w2=dense(96, 150, INT8), s2=dense(8, 96, F32)), **kw)


@pytest.mark.parametrize("status,kw", [
    (INVALID, int8(s1=None)), (INVALID, int8(s2=None)), (INVALID, int8(s1=dense(3, 2, F32))), (INVALID, int8(s1=dense(7, 300, F32))),
    (INVALID, int8(s2=dense(8, 96, BF16))), (INVALID, int8(w2=dense(96, 150, FP8))), (INVALID, int8(w1=dense(300, 200))),
    (INVALID, int8(ws=None)), (INVALID, dict(x=None)), (INVALID, dict(logits=None)), (INVALID, dict(w1=None)), (INVALID, dict(w2=None)), (INVALID, dict(out=None)),
    (INVALID, dict(top_k=0)), (INVALID, dict(top_k=9)), (INVALID, dict(normalise=2)), (INVALID, dict(logits=dense(4, 8, F32))),
    (INVALID, dict(logits=dense(5, 8, FP8))), (INVALID, dict(x=dense(5, 200, F32))), (INVALID, dict(x=dense(5, 200, F16))),
    (INVALID, dict(w1=dense(299, 200))), (INVALID, dict(w1=dense(300, 199))), (INVALID, dict(w1=dense(300, 200, INT8))),
    (INVALID, dict(w2=dense(96, 150, F16))), (INVALID, dict(w2=dense(95, 150))), (INVALID, dict(w2=dense(96, 150, FP8))),
    (INVALID, dict(w1=dense(300, 200, stack=-1))), (INVALID, dict(out=dense(5, 96, F16))), (INVALID, dict(out=dense(4, 96))),
    (INVALID, dict(s1=dense(3, 2, F32))), (INVALID, dict(s1=dense(3, 2, F32), s2=dense(1, 2, F32))), (INVALID, fp8(s1=None)),
    (INVALID, fp8(s2=None)), (INVALID, fp8(s1=dense(2, 2, F32))), (INVALID, fp8(s2=dense(1, 1, F32))), (INVALID, fp8(s1=dense(3, 2, F16))),
    (INVALID, dict(ws=None)), (INVALID, dict(ws=0x1008)), (INVALID, dict(bytes=256)), (INVALID, fp8(ws=None)),
    (INVALID, dict(x=dense(5, 200, stride=199))), (INVALID, dict(out=dense(5, 0), w2=dense(0, 150))),
    (UNSUPPORTED, dict(x=dense(65, 200), logits=dense(65, 8, F32), out=dense(65, 96))),
    (UNSUPPORTED, dict(x=dense(64, 200), logits=dense(64, 100, F32), out=dense(64, 96), top_k=17)),
    (UNSUPPORTED, dict(logits=dense(5, 1025, F32))), (UNSUPPORTED, dict(w1=dense(2 * BIG, 200), w2=dense(96, BIG)))])
def test_refusals(lib, status, kw):  # noqa: F811
    a = dict(x=dense(5, 200), logits=dense(5, 8, F32), top_k=2, normalise=1, w1=dense(300, 200), s1=None, w2=dense(96, 150), s2=None,
             out=dense(5, 96), ws=PTR, bytes=1 << 24)
    a.update(kw)
    st = lib.gmagnus_expert_layer(ref(a["x"]), ref(a["logits"]), a["top_k"], a["normalise"], ref(a["w1"]), ref(a["s1"]), ref(a["w2"]),
                                  ref(a["s2"]), ref(a["out"]), a["ws"], a["bytes"], None)
    assert st == status and lib.gmagnus_last_error()


def test_workspace_bytes(lib):  # noqa: F811
    f = lib.gmagnus_expert_layer_workspace_bytes
    assert f(1, 8, 2, 150, 96) > 0 and f(64, 8, 2, 1024, 96) >= 64 * 2 * 1024 * 2
    for bad in ((65, 8, 2, 150, 96), (4, 8, 9, 150, 96), (4, 8, 0, 150, 96), (4, 1025, 2, 150, 96), (64, 100, 17, 150, 96), (-1, 8, 2, 150, 96),
                (4, 8, 2, 0, 96), (4, 8, 2, BIG, 96), (4, 8, 2, 150, 0), (4, 8, 2, 150, 1 << 31)):
        assert f(*bad) == 0


def test_binding_refuses_host_tensors(lib):  # noqa: F811
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA tensor"):
        gm.expert_layer(x, x, 2, x[None], x[None])
