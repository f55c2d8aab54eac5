"""vlq_group_rows, vlq_gather_rows, vlq_combine_rows and its gradient against plain 64-bit forms: few and many cells (one to
three digits of the sort), dropped pairs, empty and single cells, types, odd rows, unaligned operands."""
import numpy as np
import pytest
import torch

from learn_reference import U, half_step

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def vlq():
    import paper_1901_00275_amd as vlq

    vlq.lib()
    return vlq


def group(vlq, cell, cells):
    n, w = cell.shape
    off = torch.full((cells + 1,), -7, dtype=torch.int64, device=DEV)
    place = torch.full((n, w), -7, dtype=torch.int32, device=DEV)
    source = torch.full((n * w,), -7, dtype=torch.int32, device=DEV)
    ws = torch.full((vlq.vlq_group_rows_workspace(n, w, cells),), 255, dtype=torch.uint8, device=DEV)
    vlq.vlq_group_rows(cell, n, w, cells, off, place, source, ws)
    return off, place, source


def plain(cell, cells):
    """The same by numpy's stable sort."""
    flat = cell.cpu().numpy().reshape(-1).astype(np.int64)
    kept = (flat >= 0) & (flat < cells)
    order = np.argsort(np.where(kept, flat, cells), kind="stable")
    count = int(kept.sum())
    off = np.searchsorted(flat[order[:count]], np.arange(cells + 1))
    source = np.where(np.arange(flat.size) < count, order, -1)
    place = np.full(flat.size, -1)
    place[order[:count]] = np.arange(count)
    return off, place.reshape(cell.shape), source


def check_group(vlq, cell, cells):
    got = group(vlq, cell, cells)
    for g, p in zip(got, plain(cell, cells)):
        assert np.array_equal(g.cpu().numpy(), p)
    return got


@pytest.mark.parametrize("n,w,cells", [
    (1, 1, 1), (1, 8, 8), (17, 8, 64), (63, 1, 3), (1000, 6, 128), (2048, 8, 2047), (2048, 8, 2048), (2049, 8, 100), (5000, 7, 5),
    (1, 1, 4096), (300, 64, 65536), (33333, 3, 2100), (10000, 64, 65536), (2555, 2, 4096), (20000, 30, 300), (700, 5, 1 << 24), (3, 2, 1 << 24), (1, 6, 57575), (4096, 1, 2048), (4097, 1, 2048), (1024, 4, 300000)])
def test_group(vlq, n, w, cells):
    g = torch.Generator().manual_seed(n + w + cells)
    cell = torch.randint(0, cells, (n, w), generator=g, dtype=torch.int32)
    check_group(vlq, cell.to(DEV), cells)
    # popular cells, and dropped pairs on either side of the range
    cell = (torch.rand(n, w, generator=g) ** 4 * cells).int()
    cell[torch.rand(n, w, generator=g) < 0.2] = -1
    cell[torch.rand(n, w, generator=g) < 0.1] = cells
    cell[torch.rand(n, w, generator=g) < 0.05] = 2 ** 31 - 1
    cell[torch.rand(n, w, generator=g) < 0.05] = -2 ** 31
    check_group(vlq, cell.to(DEV), cells)


@pytest.mark.parametrize("cells", [4, 3000])
def test_group_extremes(vlq, cells):
    for n in (1, 64, 65, 3000):
        for c in (0, cells - 1, -1, cells):
            off, place, source = check_group(vlq, torch.full((n, 7), c, dtype=torch.int32, device=DEV), cells)
            assert off[cells].item() == (7 * n if 0 <= c < cells else 0)


@pytest.mark.parametrize("n,w,cells", [(5, 3, 4), (700, 3, 2047), (1000, 4, 70000), (20000, 3, 300), (9000, 5, 70000), (3000, 3, 1 << 24)])
def test_nothing_is_written_past_the_buffers(vlq, n, w, cells):
    behind = lambda count, dtype: torch.full((count + 500,), 7, dtype=dtype, device=DEV)  # noqa: E731
    g = torch.Generator().manual_seed(n)
    cell = torch.randint(-1, cells, (n, w), generator=g, dtype=torch.int32).to(DEV)
    size = vlq.vlq_group_rows_workspace(n, w, cells)
    off, place, source, ws = behind(cells + 1, torch.int64), behind(n * w, torch.int32), behind(n * w, torch.int32), behind(size, torch.uint8)
    vlq.vlq_group_rows(cell, n, w, cells, off, place, source, ws)
    for buffer, count in ((off, cells + 1), (place, n * w), (source, n * w), (ws, size)):
        assert (buffer[count:] == 7).all()
    for got, want in zip((off[:cells + 1], place[:n * w].view(n, w), source[:n * w]), plain(cell, cells)):
        assert np.array_equal(got.cpu().numpy(), want)
    for t, d in ((F32, 3), (BF16, 13), (F16, 1)):
        x, y, out = torch.randn(n, d, generator=g).to(t).to(DEV), behind(n * w * d, t), behind(n * d, t)
        dy, dweight = behind(n * w * d, t), behind(n * w, F32)
        vlq.vlq_gather_rows(x, n, w, d, source, y)
        vlq.vlq_combine_rows(y, n, w, d, place, None, out)
        vlq.vlq_combine_rows_backward(x, y, n, w, d, place, None, dy, dweight)
        for buffer, count in ((y, n * w * d), (out, n * d), (dy, n * w * d), (dweight, n * w)):
            assert (buffer[count:] == 7).all()


def test_group_many_pairs(vlq):
    # tiles of the largest size
    g = torch.Generator(device=DEV).manual_seed(3)
    check_group(vlq, torch.randint(-1, 300, (600_011, 8), generator=g, device=DEV, dtype=torch.int32), 300)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,w,d,cells", [(1, 1, 1, 1), (5, 3, 7, 4), (100, 8, 64, 16), (257, 6, 96, 1000), (70, 17, 1023, 9), (1000, 2, 8, 64),
                                         (33, 64, 40, 65536), (64, 5, 2056, 7), (70, 9, 1026, 9), (50, 17, 28, 40), (41, 24, 6, 3)])
def test_rows(vlq, t, n, w, d, cells):
    g = torch.Generator().manual_seed(n + w + d)
    cell = torch.randint(0, cells, (n, w), generator=g, dtype=torch.int32)
    cell[torch.rand(n, w, generator=g) < 0.2] = -1
    if n > 3:
        cell[2] = -1  # a row that nothing comes back for
    off, place, source = group(vlq, cell.to(DEV), cells)
    kept = int(off[cells])
    x, dout = torch.randn(n, d, generator=g).to(t).to(DEV), torch.randn(n, d, generator=g).to(t).to(DEV)
    weight = torch.rand(n, w, generator=g).to(DEV)
    there = place >= 0
    weight[~there] = float("nan")  # (a dropped pair's weight is not looked at)
    y = torch.full((n * w, d), 5.0, dtype=t, device=DEV)
    vlq.vlq_gather_rows(x, n, w, d, source, y)
    assert torch.equal(y[:kept], x[(source[:kept] // w).long()])
    assert (y[kept:] == 5.0).all()  # rows behind the last pair stay as they were
    y = torch.randn(n * w, d, generator=g).to(t).to(DEV)
    y[kept:] = float("nan")
    # w products and sums in fp32, rounded once
    at = place.clamp(min=0).long()
    ys = torch.where(there[:, :, None], y[at].double(), 0.0)
    ws = torch.where(there, weight, 0.0).double()
    for wt, f in ((weight, ws), (None, there.double())):
        out = torch.full((n, d), 5.0, dtype=t, device=DEV)
        vlq.vlq_combine_rows(y, n, w, d, place, wt, out)
        want, mass = (ys * f[:, :, None]).sum(1), (ys.abs() * f[:, :, None]).sum(1)
        tol = mass * (w + 1) * U + half_step(t) * (want.abs() + mass * w * U) + (2.0 ** -25 if t == F16 else 0.0)
        assert ((out.double() - want).abs() <= tol).all()
        # the gradient
        dy = torch.full((n * w, d), 5.0, dtype=t, device=DEV)
        dweight = torch.full((n, w), 5.0, device=DEV)
        vlq.vlq_combine_rows_backward(dout, y, n, w, d, place, wt, dy, dweight)
        wanted = torch.full((n * w, d), 5.0, dtype=torch.float64, device=DEV)
        wanted[place[there].long()] = (f[:, :, None] * dout.double()[:, None, :])[there]
        err = (dy.double() - wanted).abs()
        assert (err[:kept] <= wanted[:kept].abs() * (half_step(t) + U) * 1.001 + (2.0 ** -25 if t == F16 else 0.0)).all()
        assert (dy[kept:] == 5.0).all()
        dots, mass = (ys * dout.double()[:, None, :]).sum(2), (ys * dout.double()[:, None, :]).abs().sum(2)
        assert ((dweight.double() - dots).abs() <= mass * (d + 8) * U).all()
        # each alone
        dy2, dw2 = torch.full_like(dy, 5.0), torch.full_like(dweight, 5.0)
        vlq.vlq_combine_rows_backward(dout, None, n, w, d, place, wt, dy2, None)
        vlq.vlq_combine_rows_backward(dout, y, n, w, d, place, wt, None, dw2)
        assert torch.equal(dy, dy2) and torch.equal(dweight, dw2)


@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_unaligned_rows(vlq, t):
    n, w, d, cells = 50, 4, 64, 9
    g = torch.Generator().manual_seed(1)
    cell = torch.randint(-1, cells, (n, w), generator=g, dtype=torch.int32).to(DEV)
    off, place, source = group(vlq, cell, cells)
    kept = int(off[cells])
    shift = lambda v: torch.cat([v.reshape(-1)[:1], v.reshape(-1)])[1:].view(v.shape)  # noqa: E731
    x, y0 = torch.randn(n, d, generator=g).to(t).to(DEV), torch.randn(n * w, d, generator=g).to(t).to(DEV)
    weight = torch.rand(n, w, generator=g).to(DEV)
    res = []
    for f in (lambda v: v, shift):
        y, out, dy, dw = f(torch.zeros_like(y0)), f(torch.zeros_like(x)), f(torch.zeros_like(y0)), f(torch.zeros_like(weight))
        vlq.vlq_gather_rows(f(x), n, w, d, f(source), y)
        vlq.vlq_combine_rows(f(y0), n, w, d, f(place), f(weight), out)
        vlq.vlq_combine_rows_backward(f(x), f(y0), n, w, d, f(place), f(weight), dy, dw)
        res.append((y, out, dy, dw))
    for a, b in zip(*res[:2]):
        if a.dtype == F32 and a.shape == weight.shape:  # (another order of the sums)
            assert ((a - b).abs() <= 2 * (d + 8) * U * (y0.float().abs().max() * x.float().abs().max() * d)).all()
        else:
            assert torch.equal(a, b)
    assert kept > 0


def test_more_pieces_than_threads_of_a_grid(vlq):
    # 2^24 rows of an odd size, a workgroup each; 2^28 of one value, 16 lanes each
    n, d = (1 << 24) + 3, 513
    g = torch.Generator(device=DEV).manual_seed(11)
    x = torch.randint(-30000, 30000, (n, d), generator=g, device=DEV, dtype=torch.int16).view(BF16)
    back = torch.arange(n - 1, -1, -1, device=DEV, dtype=torch.int32)
    y = torch.empty_like(x)
    vlq.vlq_gather_rows(x, n, 1, d, back, y)
    for p in (0, 1, n // 2, n - 1):
        assert torch.equal(y[p].view(torch.int16), x[n - 1 - p].view(torch.int16))
    out = torch.zeros_like(x)
    x = x.nan_to_num_()  # (combined values are sums: NaNs need not keep their bits)
    vlq.vlq_gather_rows(x, n, 1, d, back, y)
    vlq.vlq_combine_rows(y, n, 1, d, back, None, out)
    assert torch.equal(out, x)
    del x, y, out
    n = (1 << 28) + 5
    dout, y = (torch.randint(-8, 9, (n, 1), generator=g, device=DEV, dtype=torch.int8).to(F16) for _ in range(2))
    back = torch.arange(n - 1, -1, -1, device=DEV, dtype=torch.int32)
    dy, dweight = torch.empty_like(y), torch.empty(n, 1, device=DEV)
    vlq.vlq_combine_rows_backward(dout, y, n, 1, 1, back, None, dy, dweight)
    assert torch.equal(dy, dout.flip(0)) and torch.equal(dweight, (dout * y.flip(0)).float())


def test_captured_and_replayed(vlq):
    n, w, d, cells = 3000, 6, 96, 3000
    cell = torch.zeros(n, w, dtype=torch.int32, device=DEV)
    x, weight = torch.zeros(n, d, device=DEV), torch.zeros(n, w, device=DEV)
    off, place = torch.empty(cells + 1, dtype=torch.int64, device=DEV), torch.empty(n, w, dtype=torch.int32, device=DEV)
    source = torch.empty(n * w, dtype=torch.int32, device=DEV)
    y, out = torch.empty(n * w, d, device=DEV), torch.empty(n, d, device=DEV)
    ws = torch.empty(vlq.vlq_group_rows_workspace(n, w, cells), dtype=torch.uint8, device=DEV)

    def step():
        vlq.vlq_group_rows(cell, n, w, cells, off, place, source, ws)
        vlq.vlq_gather_rows(x, n, w, d, source, y)
        vlq.vlq_combine_rows(y, n, w, d, place, weight, out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator(device=DEV).manual_seed(7)
    for turn in range(4):
        cell.copy_(torch.randint(0, cells, (n, w), generator=g, device=DEV, dtype=torch.int32))
        x.copy_(torch.randn(n, d, generator=g, device=DEV))
        weight.copy_(torch.rand(n, w, generator=g, device=DEV))
        step()
        torch.cuda.synchronize()
        want = [v.clone() for v in (off, place, source, y, out)]
        for v in (off, place, source, y, out):
            v.fill_(-9)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (off, place, source, y, out)):
            assert torch.equal(a, b), turn


def test_no_rows(vlq):
    e = torch.empty(0, 3, dtype=torch.int32, device=DEV)
    off, _, _ = group(vlq, e, 5)
    assert (off == 0).all()
    z = torch.empty(0, 8, device=DEV)
    vlq.vlq_gather_rows(z, 0, 3, 8, e, z)
    vlq.vlq_combine_rows(z, 0, 3, 8, e, None, z)
    vlq.vlq_combine_rows_backward(z, z, 0, 3, 8, e, None, z, None)
