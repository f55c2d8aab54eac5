"""The sums of vlq_softmax_loss and its gradient over many rows, many centroids and many dimensions: pieces of either in every form
and type, sums that are exact in fp32 whatever their order, and large logits that leave losses and gradients to be seen."""
import math
import os
import re

import pytest
import torch

from learn_reference import softmax_loss
from test_gpu_softmax_loss import BF16, DEV, F16, F32, compare, problem, run, vlq  # noqa: F401

pytestmark = pytest.mark.gpu
SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1901_00275_amd", "csrc", "softmax_loss.hip")


def constant(name):
    with open(SOURCE) as f:
        value = re.search(rf"^#define {name} (?:\(1 << (\d+)\)|(\d+))", f.read(), re.M)
    return 1 << int(value[1]) if value[1] else int(value[2])


def wide_pieces(t, n, d, k):
    """Blocks of rows and pieces of centroids of the wide form, and whether the centroids are taken as they lie."""
    assert d > constant("NARROW_DIM" if t == F32 else "NARROW_DIM_16") and n * k > constant("FEW_PAIRS")
    rows = min(n, constant("LOSS_ROWS"))
    piece = constant("PIECE") // (-(-rows // 256) * 256) // 256 * 256
    return -(-n // rows), -(-k // piece), t != F32 and n <= constant("LIE_ROWS") and d % 8 == 0


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k,blocks,pieces", [(8492, 264, 9001, 2, 2), (4096, 264, 17000, 1, 2), (4095, 303, 33100, 1, 3), (16500, 300, 1500, 3, 1)])
def test_pieces_of_the_wide_form(vlq, t, n, d, k, blocks, pieces):  # noqa: F811
    assert wide_pieces(t, n, d, k) == (blocks, pieces, t != F32 and n <= 4096 and d % 8 == 0)
    x, c, bias, label, grad = problem(t, n, d, k, skip=0.05, out=0.02)
    label[::97] = k - 1  # (labels in the last piece, which is shorter)
    bias[k - 1] = 0.5
    compare(run(vlq, x, c, bias, 0.7, label, grad), softmax_loss(x, c, bias, 0.7, label, grad))


def whole_numbers(g, rows, d, most, t):
    return torch.randint(-most, most + 1, (rows, d), generator=g, device=DEV).to(t)


@pytest.mark.parametrize("t,n,d,k", [
    (F32, 4_300_000, 2, 4), (BF16, 300_001, 24, 64), (BF16, 1 << 27, 2, 4),  # narrow
    (F32, 30_000, 96, 1024), (F16, 30_000, 200, 1024), (BF16, 30_000, 200, 1024),
    (F32, 70_001, 264, 256), (F16, 70_001, 264, 256), (BF16, 70_001, 300, 256), (BF16, 4_000, 264, 8192),  # wide
    (F32, 9_001, 40, 64), (F16, 9_001, 40, 64), (BF16, 5_001, 1000, 16)])  # few
def test_exact_sums_over_rows(vlq, t, n, d, k):  # noqa: F811
    # Centroids of zeros, k a power of two: every probability is 1 / k, and with whole numbers for x and powers of two for the rows'
    # gradients every sum is one of multiples of 1 / (2 k) that stays below 2^23 of them.  So it has one value, in any order.
    g = torch.Generator(device=DEV).manual_seed(n + d)
    # the terms' signs are random: sums grow like sqrt(n), 6 sqrt(n) 3 most * 2 k of those multiples at most
    most = max(1, min(8, int(2 ** 23 / (6 * 3 * 2 * k * math.sqrt(n)))))
    x, c = whole_numbers(g, n, d, most, t), torch.zeros(k, d, dtype=t, device=DEV)
    label = torch.randint(-1, k, (n,), generator=g, device=DEV, dtype=torch.int32)
    label[-1] = k - 1
    grad = 2.0 ** torch.randint(-1, 2, (n,), generator=g, device=DEV)
    got = run(vlq, x, c, torch.zeros(k, device=DEV), 0.5, label, grad)
    keep = label >= 0
    w = torch.where(keep, grad, 0.0).double()
    at = torch.where(keep, label, 0).long()
    v = torch.cat([x.double() * w[:, None], w[:, None]], 1)  # (sums of whole multiples of 1 / 2: exact in 64 bits; no atomics, they would meet in k places)
    if k <= 64:
        own = torch.stack([torch.where((at == j)[:, None], v, 0.0).sum(0) for j in range(k)])
    else:
        own = torch.nn.functional.one_hot(at, k).double().t().contiguous() @ v
    both = v.sum(0) / k - own
    dc, db = both[:, :d].contiguous(), both[:, d].contiguous()
    assert float(max(db.abs().max(), dc.abs().max())) * 2 * k < 2 ** 23  # (no result is out of what this holds for)
    assert torch.equal(got["db"].double(), db)
    assert torch.equal(got["dc"], (0.5 * dc).to(t))
    assert float((dc != 0).double().mean()) > 0.9
    assert torch.equal(got["dx"], torch.zeros_like(x))
    assert float((got["loss"].double() - keep * math.log(k)).abs().max()) <= 4 * 2.0 ** -24 * math.log(k)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k", [(1000, 96, 16384), (1000, 200, 16384), (1000, 264, 16384), (4500, 300, 16384), (9000, 264, 8192), (60, 96, 16384)])
def test_exact_sums_over_centroids(vlq, t, n, d, k):  # noqa: F811
    # rows of zeros: dx is the mean of the centroids less the label's, sums of multiples of 1 / k below 2^24 of them
    g = torch.Generator(device=DEV).manual_seed(n + d)
    x, c = torch.zeros(n, d, dtype=t, device=DEV), whole_numbers(g, k, d, 1, t)
    label = torch.randint(-1, k, (n,), generator=g, device=DEV, dtype=torch.int32)
    grad = 2.0 ** torch.randint(-1, 2, (n,), generator=g, device=DEV)
    got = run(vlq, x, c, None, 2.0, label, grad)
    keep = (label >= 0)[:, None]
    C = c.double()
    assert float(C.sum(0).abs().max() + 1) * k < 2 ** 24
    dx = torch.where(keep, (C.sum(0) / k - C[label.clamp(min=0).long()]) * grad.double()[:, None], 0.0)
    assert torch.equal(got["dx"], (2.0 * dx).to(t))
    assert torch.equal(got["dc"], torch.zeros_like(c))


def seen(got, want, shares):
    """Inside the bounds, and at least such shares of what is looked for well above them."""
    compare(got, want)
    for name, share in shares.items():
        ref, tol = want[name]
        assert float((ref.abs() > 4 * tol).double().mean()) >= share, name


def far_problem(t, n, d, k):
    """Logits of hundreds; of every other row the label is no likely centroid, of the others the margin does not grow with d."""
    g = torch.Generator().manual_seed(n + d + k)
    c = torch.randn(k, d, generator=g)
    label = torch.randint(0, k, (n,), generator=g, dtype=torch.int32)
    # |c|^2 = d: a share of 1 / sqrt(d) of the label's centroid is a logit of about one standard deviation of all others, 90
    x = 90.0 * (torch.randn(n, d, generator=g) + (torch.arange(n) % 2)[:, None] * 3.0 * c[label.long()] / math.sqrt(d)) / math.sqrt(d)
    bias, grad = torch.randn(k, generator=g), (torch.rand(n, generator=g) + 0.5) / n
    return x.to(t).to(DEV), c.to(t).to(DEV), bias.to(DEV), label.to(DEV), grad.to(DEV)


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,d,k", [(130, 128, 600), (1030, 128, 1600), (1030, 160, 1600), (1000, 300, 1100), (1200, 2052, 700)])
def test_large_logits_seen(vlq, t, n, d, k):  # noqa: F811
    x, c, bias, label, grad = far_problem(t, n, d, k)
    want = softmax_loss(x, c, bias, 1.0, label, grad)
    seen(run(vlq, x, c, bias, 1.0, label, grad), want, {"loss": 0.7, "dx": 0.5, "dc": 0.35, "db": 0.35})


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k", [(5001, 2052, 61), (1500, 2052, 700), (1100, 4100, 500)])
def test_many_dimensions_seen(vlq, t, n, d, k):  # noqa: F811
    x, c, bias, label, grad = far_problem(t, n, d, k)
    x = (x.float() / 45.0).to(t)  # (logits of a few units)
    grad = grad * n  # (gradients of fp16 above its smallest steps)
    want = softmax_loss(x, c, bias, 1.0, label, grad)
    seen(run(vlq, x, c, bias, 1.0, label, grad), want, {"loss": 0.95, "dx": 0.8, "dc": 0.8, "db": 0.8})
