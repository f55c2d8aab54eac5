"""vlq_group_rows, the gather and the combination at the largest number of pairs."""
import pytest
import torch

from test_gpu_group_rows import BF16, DEV, group, vlq  # noqa: F401

pytestmark = pytest.mark.gpu


def test_most_pairs(vlq):  # noqa: F811
    # 2^31 - 1 pairs of two digits.  The order is checked as what it is: cells do not fall, pairs of one cell rise, places are the
    # inverse, an offset is where its cell begins; that leaves one order.
    n, cells = (1 << 31) - 1, 70_001
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160e9:
        pytest.skip("needs 160 GB of device memory")
    g = torch.Generator(device=DEV).manual_seed(4)
    cell = torch.empty(n, dtype=torch.int32, device=DEV).random_(-1, cells, generator=g)
    off, place, source = group(vlq, cell.view(n, 1), cells)
    place = place.view(-1)
    kept = int(off[cells])
    step, dropped, last = 1 << 28, 0, (-1, -1)
    for a in range(0, n, step):
        b = min(a + step, n)
        gone = cell[a:b] < 0
        dropped += int(gone.sum())
        assert torch.equal(place[a:b] == -1, gone)
        e = min(b, kept)
        if a < e:
            src = source[a:e].long()
            assert int(src.min()) >= 0 and int(src.max()) < n
            assert torch.equal(place[src], torch.arange(a, e, device=DEV, dtype=torch.int32))
            c = cell[src]
            assert last < (int(c[0]), int(src[0]))
            assert bool(((c[1:] > c[:-1]) | ((c[1:] == c[:-1]) & (src[1:] > src[:-1]))).all())
            last = (int(c[-1]), int(src[-1]))
        assert bool((source[max(a, kept):b] == -1).all())
    assert kept == n - dropped and off[0].item() == 0 and bool((off[1:] > off[:-1]).all())
    j = torch.arange(cells, device=DEV)
    assert torch.equal(cell[source[off[:-1]].long()].long(), j) and torch.equal(cell[source[off[1:] - 1].long()].long(), j)
    # rows of one value there and back
    x = torch.empty(n, 1, dtype=torch.int16, device=DEV).random_(-30000, 30000, generator=g).view(BF16)
    y, out = torch.zeros_like(x), torch.empty_like(x)
    vlq.vlq_gather_rows(x, n, 1, 1, source, y)
    for a in (0, kept // 2, kept - 1000):
        assert torch.equal(y[a:a + 1000].view(torch.int16), x[source[a:a + 1000].long()].view(torch.int16))
    vlq.vlq_combine_rows(y, n, 1, 1, place, None, out)
    for a in range(0, n, step):
        b = min(a + step, n)
        want = torch.where((cell[a:b] >= 0)[:, None], x[a:b], 0.0)
        assert torch.equal(out[a:b].nan_to_num(0.0), want.nan_to_num(0.0))
