"""The operators for learning cells by gradient refuse what they cannot serve, before anything touches the GPU."""
import ctypes as C

import pytest
import torch

BIG = 1 << 40


@pytest.fixture(scope="module")
def vlq():
    import os

    import paper_1901_00275_amd as vlq
    from paper_1901_00275_amd import build as vlq_build

    if not os.path.exists(vlq.LIB_PATH):
        vlq_build.build()
    return vlq


def at(i):
    """The i-th of some aligned addresses a MB apart"""
    return C.c_void_p(4096 + (i << 20))


LOSS = dict(dtype=0, x=at(0), n=10, d=8, c=at(1), k=20, bias=None, scale=1.0, label=at(2), loss=at(3), stats=at(4), grad=at(5), dx=at(6), dc=at(7),
            db=None, ws=at(8), size=BIG)


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
    dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(n=(1 << 27) + 1), dict(d=0), dict(d=16385), dict(k=0), dict(k=(1 << 24) + 1),
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
    assert loss_call(vlq, False, k=5, size=small - 1) == vlq.VLQ_EINVAL and "bytes" in vlq.vlq_last_error()
    for n, d, k in ((8000, 4000, 64), (300, 200, 100), (100_000, 128, 1000), (1, 16384, 1 << 24), (1 << 27, 1, 1)):  # the second's is enough for both
        assert L.vlq_softmax_loss_workspace(1, n, d, k, 1) >= L.vlq_softmax_loss_workspace(1, n, d, k, 0) > 0
    # the largest sizes stay within 64 bits
    assert L.vlq_softmax_loss_workspace(0, 1 << 27, 16384, 1 << 24, 1) > 0
    with pytest.raises(vlq.VlqError):
        vlq.vlq_softmax_loss_workspace(torch.float32, -1, 8, 5, False)
    with pytest.raises(ValueError):
        vlq.vlq_softmax_loss_workspace(torch.float64, 1, 8, 5, False)


def test_binding_wants_device_tensors(vlq):
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        vlq.vlq_softmax_loss(x, 4, 8, x, 4, None, 1.0, torch.zeros(4, dtype=torch.int32), None, torch.zeros(4, 2), torch.zeros(64, dtype=torch.uint8))


@pytest.mark.parametrize("change", [
    dict(n=-1), dict(w=0), dict(n=1 << 30, w=2), dict(cells=0), dict(cells=(1 << 24) + 1), dict(cell=None), dict(off=None), dict(place=None),
    dict(source=None), dict(ws=None), dict(cell=C.c_void_p(4098)), dict(off=C.c_void_p(4100)), dict(ws=C.c_void_p(4104)), dict(size=0)])
def test_group(vlq, change):
    a = dict(dict(cell=at(0), n=10, w=2, cells=5, off=at(1), place=at(2), source=at(3), ws=at(4), size=BIG), **change)
    assert vlq.lib().vlq_group_rows(a["cell"], a["n"], a["w"], a["cells"], a["off"], a["place"], a["source"], a["ws"], a["size"],
                                    None) == vlq.VLQ_EINVAL
    assert vlq.vlq_last_error() != ""


def test_group_workspace(vlq):
    L = vlq.lib()
    assert L.vlq_group_rows_workspace(-1, 1, 1) == vlq.VLQ_EINVAL and L.vlq_group_rows_workspace(1, 0, 1) == vlq.VLQ_EINVAL
    assert L.vlq_group_rows_workspace(0, 1, 1) > 0 and L.vlq_group_rows_workspace((1 << 31) - 1, 1, 1 << 24) > 0
    need = L.vlq_group_rows_workspace(1 << 20, 8, 300)
    assert L.vlq_group_rows(at(0), 1 << 20, 8, 300, at(100), at(200), at(300), at(400), need - 1, None) == vlq.VLQ_EINVAL and "bytes" in vlq.vlq_last_error()


@pytest.mark.parametrize("change", [
    dict(dtype=7), dict(n=-1), dict(w=0), dict(n=1 << 30, w=4), dict(d=0), dict(d=(1 << 20) + 1), dict(x=None), dict(index=None), dict(y=None),
    dict(x=C.c_void_p(4098)), dict(index=C.c_void_p(4097)), dict(y=C.c_void_p(4097))])
def test_rows(vlq, change):
    a = dict(dict(dtype=0, x=at(0), n=10, w=2, d=8, index=at(1), weight=None, y=at(2)), **change)
    L = vlq.lib()
    assert L.vlq_gather_rows(a["dtype"], a["x"], a["n"], a["w"], a["d"], a["index"], a["y"], None) == vlq.VLQ_EINVAL
    assert L.vlq_combine_rows(a["dtype"], a["x"], a["n"], a["w"], a["d"], a["index"], a["weight"], a["y"], None) == vlq.VLQ_EINVAL
    back = lambda dout, y, dy, dw: L.vlq_combine_rows_backward(a["dtype"], dout, y, a["n"], a["w"], a["d"], a["index"], None, dy, dw, None)  # noqa: E731
    assert back(a["x"], a["y"], at(3), at(4)) == vlq.VLQ_EINVAL
    assert L.vlq_combine_rows(0, at(0), 10, 2, 8, at(1), C.c_void_p(4098 + (2 << 20)), at(3), None) == vlq.VLQ_EINVAL
    assert L.vlq_combine_rows_backward(0, at(0), None, 10, 2, 8, at(2), None, at(3), at(4), None) == vlq.VLQ_EINVAL  # d_dweight needs d_y
    assert L.vlq_combine_rows_backward(0, at(0), at(1), 10, 2, 8, at(2), None, C.c_void_p(4098 + (3 << 20)), at(4), None) == vlq.VLQ_EINVAL


def clip_call(vlq, counts, grads, outs, dtypes=None, limit=1.0, norm=at(100), ws=at(101), size=BIG, tensors=None):
    n = len(counts)
    many = max(1, n)
    ptrs = lambda v: None if v is None else (C.c_void_p * many)(*v)  # noqa: E731
    return vlq.lib().vlq_clip_grads(n if tensors is None else tensors, (C.c_int32 * many)(*(dtypes or [0] * n)), (C.c_int64 * many)(*counts),
                                    ptrs(grads), limit, ptrs(outs), norm, ws, size, None)


def test_clip(vlq):
    bad = [
        dict(counts=[5, -1], grads=[4096, 8192], outs=None), dict(counts=[5], grads=[None], outs=None), dict(counts=[5], grads=[4098], outs=None),
        dict(counts=[5], grads=[4096], outs=[None]), dict(counts=[5], grads=[4096], outs=[8194]), dict(counts=[5], grads=None, outs=None),
        dict(counts=[5], grads=[4096], outs=None, dtypes=[3]), dict(counts=[5], grads=[4096], outs=None, limit=0.0),
        dict(counts=[5], grads=[4096], outs=None, limit=-1.0), dict(counts=[5], grads=[4096], outs=None, limit=float("nan")),
        dict(counts=[5], grads=[4096], outs=None, ws=None), dict(counts=[5], grads=[4096], outs=None, size=8),
        dict(counts=[5], grads=[4096], outs=None, norm=C.c_void_p(4098)), dict(counts=[5], grads=[4096], outs=None, tensors=-1),
        dict(counts=[1 << 47, 1 << 48], grads=[4096, 8192], outs=None),
        # overlaps: the same tensor twice, an output over its own input's middle, over another input, over another output
        dict(counts=[5, 5], grads=[4096, 4096], outs=[4096, 4096]), dict(counts=[5], grads=[4096], outs=[4100]),
        dict(counts=[5, 5], grads=[4096, 8192], outs=[4096, 4112]), dict(counts=[5, 5], grads=[4096, 8192], outs=[12288, 12300])]
    for kw in bad:
        assert clip_call(vlq, **kw) == vlq.VLQ_EINVAL, kw
        assert vlq.vlq_last_error() != ""
    many = 500
    assert clip_call(vlq, [4] * many, [4096 + 16 * i for i in range(many)], [4096 + 16 * (many - i) for i in range(many)]) == vlq.VLQ_EINVAL


def test_clip_workspace(vlq):
    L = vlq.lib()
    assert L.vlq_clip_grads_workspace(-1, None) == vlq.VLQ_EINVAL and L.vlq_clip_grads_workspace(1, None) == vlq.VLQ_EINVAL
    assert L.vlq_clip_grads_workspace(0, None) > 0


def test_overlaps(vlq):
    inside = lambda i: C.c_void_p(4096 + (i << 20) + 64)  # noqa: E731
    for change in (dict(loss=at(0)), dict(loss=inside(1)), dict(stats=at(2)), dict(ws=at(0)), dict(ws=C.c_void_p(4096 + (8 << 20)), x=inside(8))):
        assert loss_call(vlq, False, **change) == vlq.VLQ_EINVAL and "overlap" in vlq.vlq_last_error(), change
    for change in (dict(dx=at(0)), dict(dc=inside(1)), dict(dx=inside(7)), dict(db=inside(6)), dict(dx=at(5)), dict(dx=at(4)), dict(ws=at(7))):
        assert loss_call(vlq, True, **change) == vlq.VLQ_EINVAL and "overlap" in vlq.vlq_last_error(), change
    L = vlq.lib()
    assert L.vlq_group_rows(at(0), 10, 2, 5, at(1), at(2), inside(2), at(4), BIG, None) == vlq.VLQ_EINVAL
    assert L.vlq_gather_rows(0, at(0), 10, 2, 8, at(1), inside(0), None) == vlq.VLQ_EINVAL
    assert L.vlq_combine_rows(0, at(0), 10, 2, 8, at(1), None, inside(0), None) == vlq.VLQ_EINVAL
    assert L.vlq_combine_rows_backward(0, at(0), at(1), 10, 2, 8, at(2), None, inside(1), None, None) == vlq.VLQ_EINVAL
    assert "overlap" in vlq.vlq_last_error()
    assert clip_call(vlq, [5], [4096], [8192], norm=C.c_void_p(8196), ws=at(3)) == vlq.VLQ_EINVAL
    assert clip_call(vlq, [5], [4096], [8192], norm=at(1), ws=C.c_void_p(4096)) == vlq.VLQ_EINVAL
    for change in (dict(ws=C.c_void_p(4096)), dict(norm=C.c_void_p(4100)), dict(norm=at(101))):  # the norm alone
        assert clip_call(vlq, [5], [4096], None, **change) == vlq.VLQ_EINVAL and "overlap" in vlq.vlq_last_error(), change
