"""vlq_softmax_loss and its gradient where their range or their bits could end: probabilities whose terms cancel, biases that take up
the products, in every form and type, against the formulas in 64 bits."""

import math

import pytest
import torch

from learn_reference import SUB, U, half_step, softmax_loss
from test_gpu_softmax_loss import BF16, F16, F32, DEV, problem, run, vlq  # noqa: F401

pytestmark = pytest.mark.gpu


def within(got, want, name):
    """Everything inside its bound, and the bound far below what is looked for."""
    ref, tol = want[name]
    err = (got[name].double() - ref).abs()
    assert (err <= tol).all(), f"{name}: off by up to {float((err / tol).max()):.3g} bounds"
    assert float((ref.abs() > 4 * tol).double().mean()) > 0.5, f"{name}: the bound says little"


def bounds(x, c, bias, scale, label, grad):
    """The bounds of fp32 operands, with the outputs rounded once to the operands' type: all between is held to 22 bits or more."""
    want = softmax_loss(x.float(), c.float(), bias, scale, label, grad)
    for name in ("dx", "dc"):
        ref, tol = want[name]
        want[name] = ref, tol + half_step(x.dtype) * (ref.abs() + tol) + (2.0 ** -25 if x.dtype == F16 else 0.0)
    return want


@pytest.mark.parametrize("t", [F32, F16, BF16])
# narrow, of 16-bit values up to 256 dimensions; wide from images and with the centroids as they lie
@pytest.mark.parametrize("d", [96, 200, 300, 304])
def test_terms_that_cancel(vlq, t, d):  # noqa: F811
    # Operands around 30, probabilities of 1 / k all but alike, every label equally often: the rounding of one probability to
    # eleven bits (32.768 of 2^15 is off by 4e-4 of itself) is that of all, and the sums are the spread around the mean alone
    n, k, scale = 2000, 1000, 2.0 ** -26
    g = torch.Generator().manual_seed(d)
    x, c = ((30.0 + torch.randn(v, d, generator=g)).to(t).to(DEV) for v in (n, k))
    label = (torch.randperm(n, generator=g) % k).int().to(DEV)
    up = 2.0 ** 26  # (gradients near one, in fp16 as well)
    grad = torch.full((n,), up, device=DEV)
    got = run(vlq, x, c, torch.zeros(k, device=DEV), scale, label, grad)
    want = bounds(x, c, torch.zeros(k, device=DEV), scale, label, grad)
    for name in ("dx", "dc"):
        within(got, want, name)


# the gradients' forms: few; narrow, of 16-bit values also beyond 128 dimensions; wide from images and with the centroids as they lie
FORMS = [(70, 40, 300), (900, 96, 1500), (900, 200, 1500), (1000, 300, 1100), (1000, 304, 1100)]


def uniform(x, c, scale, label, grad):
    """dx, dc, db where every probability is 1 / k, and their bounds: 1 / k is a sum of ones and two roundings, a product of it two
    more; G as two fp16 parts; the sums on the matrix cores."""
    t, (n, d), k = x.dtype, x.shape, c.shape[0]
    G = torch.full((n, k), 1.0 / k, dtype=torch.float64, device=DEV)
    G[torch.arange(n, device=DEV), label.long()] -= 1.0
    G *= grad.double()[:, None]
    X, Cc = x.double(), c.double()
    off = lambda N: (N / 4 + 64) * U + 24 * U + 2.0 ** -22  # noqa: E731  (8 U of them for the parts of fp32 operands)
    top = float(grad.abs().max())
    low = 2.0 ** -39  # of the largest of the matrix
    out = {"dx": scale * (G @ Cc), "dc": scale * (G.t().contiguous() @ X), "db": G.sum(0)}
    tol = {"dx": abs(scale) * (G.abs() @ Cc.abs() * off(k) + SUB * grad.double().abs()[:, None] * Cc.abs().sum(0) + G.abs().sum(1, keepdim=True) * low * Cc.abs().max()),
           "dc": abs(scale) * (G.abs().t().contiguous() @ X.abs() * off(n) + SUB * top * X.abs().sum(0) + G.abs().sum(0)[:, None] * low * X.abs().max()),
           "db": G.abs().sum(0) * off(n)}
    for name in ("dx", "dc"):
        tol[name] = tol[name] + half_step(t) * (out[name].abs() + tol[name]) + (2.0 ** -25 if t == F16 else 0.0)
    return {name: (out[name], tol[name]) for name in out}


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k", FORMS)
def test_bias_that_takes_up_the_products(vlq, t, n, d, k):  # noqa: F811
    # all centroids masked alike by a finite value next to which logits of up to some ten vanish (in 64 bits as well): the
    # loss is log k, every probability 1 / k
    x, c, _, label, _ = problem(t, n, d, k, spread=4.0)
    bias = torch.full((k,), -2.0 ** 100, device=DEV)
    grad = torch.linspace(0.5, 1.5, n, device=DEV)
    got = run(vlq, x, c, bias, 1.0, label, grad)
    assert float((got["loss"].double() - math.log(k)).abs().max()) <= 8 * U * math.log(k)
    want = uniform(x, c, 1.0, label, grad)
    for name in ("dx", "dc", "db"):
        within(got, want, name)


LOWEST = torch.finfo(F32).min


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k", FORMS)
def test_lowest_bias(vlq, t, n, d, k):  # noqa: F811
    x, c, bias, label, grad = problem(t, n, d, k)
    # of every third centroid, the labels of many rows among them: such a centroid has the probability that a bias of -60
    # leaves (1e-26), and a row of its label a loss next to which nothing shows
    mask = torch.arange(k, device=DEV) % 3 == 0
    want = softmax_loss(x, c, torch.where(mask, -60.0, bias), 0.7, label, grad)
    got = run(vlq, x, c, torch.where(mask, LOWEST, bias), 0.7, label, grad)
    of = mask[label.long()]
    assert of.any() and not of.all()
    assert torch.equal(got["loss"][of], torch.full_like(got["loss"][of], -LOWEST))
    ref, tol = want["loss"]
    assert ((got["loss"].double() - ref).abs() <= tol)[~of].all()
    for name in ("dx", "dc", "db"):
        ref, tol = want[name]
        assert ((got[name].double() - ref).abs() <= tol).all(), name
    # of all: the probabilities are alike
    got = run(vlq, x, c, torch.full_like(bias, LOWEST), 0.7, label, grad)
    assert float((got["loss"].double() - math.log(k)).abs().max()) <= 8 * U * math.log(k)
    for name, (ref, tol) in uniform(x, c, 0.7, label, grad).items():
        assert ((got[name].double() - ref).abs() <= tol).all(), name
    # the largest, of one: it has everything
    bias[5], label[3] = -LOWEST, 5
    got = run(vlq, x, c, bias, 0.7, label, grad)
    assert got["loss"][3].item() == 0 and (got["dx"][3] == 0).all()
    assert all(v.isfinite().all() for v in got.values()) and (got["loss"][label != 5] > 2.3e38).all()


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("e", [-118, -100, 110])
@pytest.mark.parametrize("n,d,k", FORMS + [(900, 96, 40), (3000, 130, 5000)])
def test_gradients_of_any_size(vlq, t, e, n, d, k):  # noqa: F811
    # the rows' gradients near either end of fp32's range, what comes of them inside it
    x, c, bias, label, grad = problem(t, n, d, k)
    grad = n * grad * 2.0 ** e
    got, want = run(vlq, x, c, bias, 0.7, label, grad), softmax_loss(x, c, bias, 0.7, label, grad)
    for name in ("dx", "dc", "db"):
        ref, tol = want[name]
        if t == BF16 and name != "db":
            tol = tol + 2.0 ** -134  # (half its smallest step)
        assert ((got[name].double() - ref).abs() <= tol).all(), name


def test_more_sums_than_threads_of_a_grid(vlq):  # noqa: F811
    # 2^34 values of dc, added up over two blocks of rows, four a thread
    n, d, k = 8192 + 5, 16384, (1 << 20) + 77
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 225e9:
        pytest.skip("needs 225 GB of device memory")
    g = torch.Generator(device=DEV).manual_seed(3)
    c = torch.empty(k, d, dtype=BF16, device=DEV).normal_(generator=g)
    x = torch.empty(n, d, device=DEV).normal_(generator=g).mul_(d ** -0.5).to(BF16)
    label = torch.randint(0, k, (n,), generator=g, device=DEV, dtype=torch.int32)
    label[-1] = k - 1
    grad = torch.rand(n, generator=g, device=DEV) + 0.5
    loss, stats, dc = torch.empty(n, device=DEV), torch.empty(n, 2, device=DEV), torch.full((k, d), 7.0, dtype=BF16, device=DEV)
    ws = torch.empty(max(vlq.vlq_softmax_loss_workspace(BF16, n, d, k, b) for b in (0, 1)), dtype=torch.uint8, device=DEV)
    vlq.vlq_softmax_loss(x, n, d, c, k, None, 1.0, label, loss, stats, ws)
    vlq.vlq_softmax_loss_backward(x, n, d, c, k, None, 1.0, label, stats, grad, None, dc, None, ws)
    del ws
    some = torch.cat([torch.arange(3, device=DEV), label[:4].long(), torch.arange(k - 200, k, device=DEV)])
    X, lse = x.double(), math.log(2) * stats[:, 0].double() + torch.log(stats[:, 1].double())
    p = torch.exp(X @ c[some].double().t().contiguous() - lse[:, None])
    G = (p - (label.long()[:, None] == some[None, :]).double()) * grad.double()[:, None]
    ref = G.t().contiguous() @ X
    # p: logits of 16 384 products (the sum's roundings, next to their sizes of up to |x||c|) and of the statistics; G in two parts; the
    # sums over the rows
    size = float(X.norm(dim=1).max() * c[some].double().norm(dim=1).max())
    off = 2 * size * (d / 4 + 64) * U + 2.0 ** -22 + (n / 4 + 64) * U
    tol = (G.abs().t().contiguous() @ X.abs()) * off + SUB * float(grad.max()) * X.abs().sum(0)
    assert ((dc[some].double() - ref).abs() <= tol + half_step(BF16) * (ref.abs() + tol)).all()


@pytest.mark.parametrize("t", [F32, BF16])
# powers of two of x, c and the scale: logits stay ordinary, what is on the way there, the gradients and the images' scales do not
@pytest.mark.parametrize("ex,ec,es", [(-60, -60, 118), (55, 55, -108), (-118, 0, 112), (0, -118, 112), (100, -100, 0)])
@pytest.mark.parametrize("n,d,k", FORMS)
def test_operands_of_any_size(vlq, t, ex, ec, es, n, d, k):  # noqa: F811
    x, c, bias, label, grad = problem(t, n, d, k)
    x, c = x * 2.0 ** ex, c * 2.0 ** ec
    scale = 2.0 ** (es if ex + ec + es >= -6 else -(ex + ec))
    got, want = run(vlq, x, c, bias, scale, label, grad), softmax_loss(x, c, bias, scale, label, grad)
    for name in ("loss", "dx", "dc", "db"):
        ref, tol = want[name]
        # The sums of G x and G c are fp32 numbers before the scale: of operands around 2^-121 and G around 2^-18 they are below the
        # normal range, where each product and each part of a sum is off by half a step, 2^-150, and sums of steps are exact.
        if name in ("dx", "dc"):
            tol = tol + ((k if name == "dx" else n) + 64) * 2.0 ** -150 * scale + (2.0 ** -134 if t == BF16 else 0.0)
        assert ((got[name].double() - ref).abs() <= tol).all(), name
