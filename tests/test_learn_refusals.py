"""The operators for learning cells by gradient refuse what they cannot serve, before anything touches the GPU."""
import ctypes as C

import pytest
import torch

P = C.c_void_p(4096)  # an aligned address that no refused call looks at
BIG = 1 << 40


@pytest.fixture(scope="module")
def vlq():
    import os

    import paper_1901_00275_amd as vlq
    from paper_1901_00275_amd import build as vlq_build

    if not os.path.exists(vlq.LIB_PATH):
        vlq_build.build()
    return vlq


LOSS = dict(dtype=0, x=P, n=10, d=8, c=P, k=20, bias=None, scale=1.0, label=P, loss=P, stats=P, grad=P, dx=P, dc=P, db=None, ws=P, size=BIG)


def loss_call(vlq, backward, **change):
    a = dict(LOSS, **change)
    L = vlq.lib()
    if backward:
        return L.vlq_softmax_loss_backward(a["dtype"], a["x"], a["n"], a["d"], a["c"], a["k"], a["bias"], a["scale"], a["label"], a["stats"],
                                           a["grad"], a["dx"], a["dc"], a["db"], a["ws"], a["size"], None)
    return L.vlq_softmax_loss(a["dtype"], a["x"], a["n"], a["d"], a["c"], a["k"], a["bias"], a["scale"], a["label"], a["loss"], a["stats"],
                              a["ws"], a["size"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=16385), dict(k=0), dict(k=(1 << 24) + 1),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(x=None), dict(c=None), dict(label=None), dict(stats=None), dict(ws=None),
    dict(x=C.c_void_p(4098)), dict(c=C.c_void_p(4097)), dict(bias=C.c_void_p(4098)), dict(label=C.c_void_p(4097)),
    dict(ws=C.c_void_p(4096 + 128)), dict(size=100), dict(size=-1), dict(dtype=1, x=C.c_void_p(4097))])
def test_loss(vlq, backward, change):
    assert loss_call(vlq, backward, **change) == vlq.VLQ_EINVAL
    assert vlq.vlq_last_error() != ""


def test_loss_backward_outputs(vlq):
    assert loss_call(vlq, True, grad=None) == vlq.VLQ_EINVAL
    assert loss_call(vlq, True, dx=C.c_void_p(4098)) == vlq.VLQ_EINVAL
    assert loss_call(vlq, True, db=C.c_void_p(4098)) == vlq.VLQ_EINVAL
    assert loss_call(vlq, True, dx=None, dc=None, db=None) == vlq.VLQ_OK  # nothing asked for, nothing done


def test_loss_workspace(vlq):
    L = vlq.lib()
    assert L.vlq_softmax_loss_workspace(0, 10, 0, 5, 0) == vlq.VLQ_EINVAL
    assert L.vlq_softmax_loss_workspace(5, 10, 8, 5, 0) == vlq.VLQ_EINVAL
    assert L.vlq_softmax_loss_workspace(0, 0, 8, 5, 0) > 0 and L.vlq_softmax_loss_workspace(1, 0, 8, 5, 1) > 0
    assert loss_call(vlq, False, n=0, x=None, label=None, stats=None) == vlq.VLQ_OK  # no rows, nothing done
    small, large = (L.vlq_softmax_loss_workspace(0, 10, 8, 5, b) for b in (0, 1))
    assert 0 < small < large
    assert L.vlq_softmax_loss(0, P, 10, 8, P, 5, None, 1.0, P, P, P, P, small - 1, None) == vlq.VLQ_EINVAL
    # the largest sizes stay within 64 bits
    assert L.vlq_softmax_loss_workspace(0, (1 << 31) - 1, 16384, 1 << 24, 1) > 0
    with pytest.raises(vlq.VlqError):
        vlq.vlq_softmax_loss_workspace(torch.float32, -1, 8, 5, False)
    with pytest.raises(ValueError):
        vlq.vlq_softmax_loss_workspace(torch.float64, 1, 8, 5, False)


def test_binding_wants_device_tensors(vlq):
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        vlq.vlq_softmax_loss(x, 4, 8, x, 4, None, 1.0, torch.zeros(4, dtype=torch.int32), None, torch.zeros(4, 2), torch.zeros(64, dtype=torch.uint8))
