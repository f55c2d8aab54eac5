"""vlq_softmax_loss and its gradient against the formulas in 64 bits: types, odd sizes, rows and centroids that do not count,
pieces of rows and of centroids, unaligned operands, captured and replayed calls, refusals."""
import math

import pytest
import torch

from learn_reference import check, softmax_loss

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def vlq():
    import paper_1901_00275_amd as vlq

    vlq.lib()
    return vlq


def problem(t, n, d, k, seed=0, spread=1.0, bias=True, skip=0.0, out=0.0, mean=0.0):
    g = torch.Generator().manual_seed(1000 * seed + n + 7 * d + 13 * k)
    c = torch.randn(k, d, generator=g) + mean
    label = torch.randint(0, k, (n,), generator=g, dtype=torch.int32)
    x = spread * (torch.randn(n, d, generator=g) + 0.5 * c[label.long()]) / math.sqrt(d)
    label = torch.where(torch.rand(n, generator=g) < skip, torch.full_like(label, -1), label)
    b = torch.randn(k, generator=g) if bias else None
    if out:
        b = torch.where(torch.rand(k, generator=g) < out, torch.full_like(b, -math.inf), b)
    grad = torch.randn(n, generator=g) / max(n, 1)
    dev = lambda v, t=None: None if v is None else v.to(t or v.dtype).to(DEV)  # noqa: E731
    return dev(x, t), dev(c, t), dev(b), dev(label), dev(grad)


def run(vlq, x, c, bias, scale, label, grad, what=("dx", "dc", "db"), stream=None):
    (n, d), k = x.shape, c.shape[0]
    loss, stats = torch.full((n,), 7.0, device=DEV), torch.full((n, 2), 7.0, device=DEV)
    ws = torch.full((vlq.vlq_softmax_loss_workspace(x.dtype, n, d, k, 0),), 255, dtype=torch.uint8, device=DEV)  # (NaNs wherever it is read unwritten)
    vlq.vlq_softmax_loss(x, n, d, c, k, bias, scale, label, loss, stats, ws, stream)
    if grad is None:
        return {"loss": loss, "stats": stats}
    ws = torch.full((vlq.vlq_softmax_loss_workspace(x.dtype, n, d, k, 1),), 255, dtype=torch.uint8, device=DEV)
    out = {"loss": loss, "stats": stats,
           "dx": torch.full((n, d), 7.0, dtype=x.dtype, device=DEV) if "dx" in what else None,
           "dc": torch.full((k, d), 7.0, dtype=x.dtype, device=DEV) if "dc" in what else None,
           "db": torch.full((k,), 7.0, device=DEV) if "db" in what else None}
    vlq.vlq_softmax_loss_backward(x, n, d, c, k, bias, scale, label, stats, grad, out["dx"], out["dc"], out["db"], ws, stream)
    return out


def compare(got, want, names=("loss", "dx", "dc", "db")):
    for name in names:
        check(got[name], want[name], name)


SHAPES = [(1, 1, 1), (1, 96, 300), (3, 7, 2), (64, 32, 256), (65, 33, 257), (255, 96, 1000), (257, 128, 513), (300, 130, 1025),
          (40, 520, 77), (17, 1027, 515), (1000, 64, 5000), (33, 48, 65537), (9, 200, 70001), (129, 100, 9000), (700, 136, 1100), (2100, 500, 1001), (900, 264, 5003), (1500, 192, 4100),
          (1000, 128, 3000), (2049, 31, 1500), (1200, 1027, 515), (3000, 130, 1025), (1111, 520, 777), (7, 300, 33), (5000, 129, 5), (2, 64, 40000), (5001, 2052, 61), (1300, 217, 1111), (1200, 256, 1400), (1131, 257, 1100), (300, 193, 9000)]


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k", SHAPES)
def test_against_64_bits(vlq, t, n, d, k):
    x, c, bias, label, grad = problem(t, n, d, k)
    compare(run(vlq, x, c, bias, 0.7, label, grad), softmax_loss(x, c, bias, 0.7, label, grad))


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,d,k", [(1, 40, 100), (200, 96, 700), (513, 200, 300), (700, 96, 1500), (1513, 200, 1300), (1000, 300, 1100)])
def test_no_bias_negative_scale(vlq, t, n, d, k):
    x, c, _, label, grad = problem(t, n, d, k, bias=False, spread=3.0)
    compare(run(vlq, x, c, None, -1.3, label, grad), softmax_loss(x, c, None, -1.3, label, grad))


@pytest.mark.parametrize("n,d,k", [(300, 96, 900), (40, 200, 700), (900, 96, 1900), (900, 232, 1500), (1400, 328, 2600)])
@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_rows_and_centroids_that_do_not_count(vlq, t, n, d, k):
    x, c, bias, label, grad = problem(t, n, d, k, skip=0.3, out=0.3)
    label[5], label[6] = k, 2 ** 31 - 1  # (outside as well)
    label[7] = int(torch.nonzero(torch.isneginf(bias))[0])  # (the label was taken out)
    want = softmax_loss(x, c, bias, 0.7, label, grad)
    dead, gone = (label < 0) | (label >= k), torch.isneginf(bias)
    x[dead], c[gone] = math.nan, math.inf  # what does not count may hold anything
    got = run(vlq, x, c, bias, 0.7, label, grad)
    compare(got, want)
    assert math.isinf(got["loss"][7].item()) and (got["loss"][dead] == 0).all() and (got["dx"][dead] == 0).all()


@pytest.mark.parametrize("n,d,k", [(20, 64, 300), (300, 64, 3000), (1000, 160, 2000), (1000, 300, 1100)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_nothing_left(vlq, t, n, d, k):
    x, c, bias, label, grad = problem(t, n, d, k)
    bias.fill_(-math.inf)
    got = run(vlq, x, c, bias, 1.0, label, grad)
    assert torch.isposinf(got["loss"]).all()
    assert all((got[v] == 0).all() for v in ("dx", "dc", "db"))
    label.fill_(-1)  # no row counts
    bias.fill_(0.0)
    got = run(vlq, x, c, bias, 1.0, label, grad)
    assert all((got[v] == 0).all() for v in ("loss", "dx", "dc", "db"))


@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_pieces_of_rows_and_centroids(vlq, t):
    # more rows than go through the products together, more centroids than P is kept for at a time
    n, d, k = 8192 + 300, 40, 4096 + 600
    x, c, bias, label, grad = problem(t, n, d, k, skip=0.05)
    compare(run(vlq, x, c, bias, 1.0, label, grad), softmax_loss(x, c, bias, 1.0, label, grad))


def test_millions_of_rows(vlq):
    # more blocks of 64 rows than a grid has in its second dimension; and more rows than a piece, in the narrow form
    for t, n, d, k in ((F32, 4_300_000, 2, 3), (BF16, 300_001, 24, 40)):
        x, c, bias, label, grad = problem(t, n, d, k, skip=0.1)
        compare(run(vlq, x, c, bias, 1.0, label, grad), softmax_loss(x, c, bias, 1.0, label, grad))


def test_most_rows_and_most_centroids(vlq):
    g = torch.Generator(device=DEV).manual_seed(5)
    for n, d, k in ((1 << 27, 2, 3), (33, 3, 1 << 24)):
        x, c = (torch.randn(v, d, generator=g, device=DEV).to(BF16) for v in (n, k))
        label = torch.randint(-1, k, (n,), generator=g, device=DEV, dtype=torch.int32)
        label[-1] = k - 1
        bias, grad = torch.randn(k, generator=g, device=DEV), torch.randn(n, generator=g, device=DEV)
        compare(run(vlq, x, c, bias, 1.0, label, grad), softmax_loss(x, c, bias, 1.0, label, grad))


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("n,d,k", [(70, 40, 300), (70, 140, 300), (900, 40, 1500), (900, 140, 2100), (1000, 300, 1100)])
def test_gradients_that_are_not_finite(vlq, t, bad, n, d, k):
    # a row's own dx, and what is summed over the rows: whether other rows have gradients or not
    x, c, bias, label, grad = problem(t, n, d, k)
    for others in (1.0, 0.0):
        grad = grad * others
        grad[7] = bad
        got, ref = run(vlq, x, c, bias, 1.0, label, grad), run(vlq, x, c, bias, 1.0, label, torch.where(grad == grad[7], 0.0, torch.nan_to_num(grad, 0.0)))
        assert not got["dx"][7].isfinite().any()
        for name in ("dc", "db"):
            assert not got[name].isfinite().any(), name
        rest = torch.arange(n, device=DEV) != 7
        assert torch.equal(got["dx"][rest], ref["dx"][rest])


SIZES = [(130, 128, 600), (1030, 128, 1600), (1030, 160, 1600), (1000, 300, 1100)]  # of each form of the gradients


@pytest.mark.parametrize("n,d,k", SIZES)
@pytest.mark.parametrize("t", [F32, BF16])
def test_large_and_small_logits(vlq, t, n, d, k):
    # logits in the hundreds, all but one probability vanish; and descriptors with a mean far above their spread
    x, c, bias, label, grad = problem(t, n, d, k, spread=60.0)
    compare(run(vlq, x, c, bias, 1.0, label, grad), softmax_loss(x, c, bias, 1.0, label, grad))
    x, c, bias, label, grad = problem(t, n, d, k, mean=30.0)
    compare(run(vlq, x, c, bias, 0.02, label, grad), softmax_loss(x, c, bias, 0.02, label, grad))


@pytest.mark.parametrize("n,d,k", SIZES)
def test_rows_of_uneven_size(vlq, n, d, k):
    # rows 24 binades apart keep their own scale forward; the gradients are relative to the largest
    x, c, bias, label, grad = problem(F32, n, d, k)
    x[::3] *= 2.0 ** -24
    c[::7] *= 2.0 ** -10
    compare(run(vlq, x, c, bias, 1.0, label, grad), softmax_loss(x, c, bias, 1.0, label, grad))


@pytest.mark.parametrize("n", [20, 70])
@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_unaligned_operands(vlq, t, n):
    # one value past a 16-byte boundary, with a dimension that would allow wide loads
    d, k = 64, 300
    x, c, bias, label, grad = problem(t, n, d, k)
    shift = lambda v: torch.cat([v.reshape(-1)[:1], v.reshape(-1)])[1:].view(v.shape)  # noqa: E731
    xs, cs, bs, ls, gs = map(shift, (x, c, bias, label, grad))
    assert xs.data_ptr() % 16 and torch.equal(xs, x)
    one, two = run(vlq, x, c, bias, 1.0, label, grad), run(vlq, xs, cs, bs, 1.0, ls, gs)
    for name in one:
        assert torch.equal(one[name], two[name]), name


@pytest.mark.parametrize("n,d,k", SIZES + [(70, 66, 300), (70, 65, 300)])
@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_unaligned_operands_against_64_bits(vlq, t, n, d, k):
    x, c, bias, label, grad = problem(t, n, d, k)
    for by in (1, 2, 4):
        shift = lambda v: torch.cat([v.reshape(-1)[:by], v.reshape(-1)])[by:].view(v.shape)  # noqa: E731
        ops = [shift(v) for v in (x, c, bias)]
        compare(run(vlq, *ops, 1.0, label, grad), softmax_loss(x, c, bias, 1.0, label, grad))


@pytest.mark.parametrize("n,d,k", [(300, 160, 700), (600, 96, 1000), (1500, 160, 1100), (1000, 300, 1100)])
@pytest.mark.parametrize("what", [("dx",), ("dc",), ("db",), ("dx", "db")])
def test_some_gradients_alone(vlq, what, n, d, k):
    x, c, bias, label, grad = problem(BF16, n, d, k)
    whole, part = run(vlq, x, c, bias, 1.0, label, grad), run(vlq, x, c, bias, 1.0, label, grad, what)
    for name in what:
        assert torch.equal(whole[name], part[name]), name


def test_against_differences(vlq):
    # the gradient along random directions is the central difference of the 64-bit loss: its error is h^2 / 6 of the third
    # derivative, which is below 2 (2 s |v| max|c|)^3 along a direction v of one row
    n, d, k, h, s = 5, 16, 40, 1e-4, 0.9
    x, c, bias, label, grad = problem(F32, n, d, k)
    got, want = run(vlq, x, c, bias, s, label, grad), softmax_loss(x, c, bias, s, label, grad)
    total = lambda X, Cc, B: (softmax_loss(X, Cc, B, s, label)["loss"][0] * grad.double()).sum()  # noqa: E731
    g = torch.Generator().manual_seed(5)
    for name, at in (("dx", 0), ("dc", 1), ("db", 2)):
        ops = [x.double(), c.double(), bias.double()]
        v = torch.randn(ops[at].shape, generator=g, dtype=torch.float64).to(DEV)
        v /= v.norm()
        up, down = list(ops), list(ops)
        up[at], down[at] = ops[at] + h * v, ops[at] - h * v
        # (64-bit operands: the reference's own bounds are not looked at)
        diff = (total(*up) - total(*down)) / (2 * h)
        third = 2 * (2 * s * max(1.0, c.abs().max().item() * d ** 0.5, x.abs().max().item() * d ** 0.5)) ** 3 * grad.abs().sum().item()
        tol = h * h / 6 * third + (want[name][1] * v.abs()).sum().item() + 1e-11
        assert abs((got[name].double() * v).sum().item() - diff.item()) <= tol, name


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,d,k", [(3, 5, 7), (33, 77, 3000), (1100, 201, 77), (300, 65, 3001), (1030, 160, 1601), (1030, 301, 1601), (8300, 130, 9001)])
def test_nothing_is_written_past_the_buffers(vlq, t, n, d, k):
    x, c, bias, label, grad = problem(t, n, d, k)
    behind = lambda count, dtype: torch.full((count + 1000,), 7, dtype=dtype, device=DEV)  # noqa: E731
    loss, stats, dx, dc, db = behind(n, F32), behind(2 * n, F32), behind(n * d, t), behind(k * d, t), behind(k, F32)
    sizes = [vlq.vlq_softmax_loss_workspace(t, n, d, k, b) for b in (0, 1)]
    ws = [behind(s, torch.uint8) for s in sizes]
    vlq.vlq_softmax_loss(x, n, d, c, k, bias, 1.0, label, loss, stats, ws[0])
    vlq.vlq_softmax_loss_backward(x, n, d, c, k, bias, 1.0, label, stats, grad, dx, dc, db, ws[1])
    for buffer, count in ((loss, n), (stats, 2 * n), (dx, n * d), (dc, k * d), (db, k), (ws[0], sizes[0]), (ws[1], sizes[1])):
        assert (buffer[count:] == 7).all()
    want = softmax_loss(x, c, bias, 1.0, label, grad)
    compare({"loss": loss[:n], "dx": dx[:n * d].view(n, d), "dc": dc[:k * d].view(k, d), "db": db[:k]}, want)


def test_stats_give_the_log_sum(vlq):
    x, c, bias, label, _ = problem(F32, 100, 96, 3000)
    got, want = run(vlq, x, c, bias, 1.0, label, None), softmax_loss(x, c, bias, 1.0, label)
    lse = math.log(2) * got["stats"][:, 0].double() + torch.log(got["stats"][:, 1].double())
    check(lse, (want["m"] + torch.log(want["z"]), want["loss"][1]), "log sum")


@pytest.mark.parametrize("n,d,k", [(300, 96, 2000), (40, 200, 300), (5000, 150, 7), (1000, 160, 1700)])
def test_captured_and_replayed(vlq, n, d, k):
    x, c, bias, label, grad = problem(F32, n, d, k)
    ws = torch.empty(vlq.vlq_softmax_loss_workspace(F32, n, d, k, 1), dtype=torch.uint8, device=DEV)
    loss, stats = torch.empty(n, device=DEV), torch.empty(n, 2, device=DEV)
    dx, dc, db = torch.empty_like(x), torch.empty_like(c), torch.empty_like(bias)

    def step():
        vlq.vlq_softmax_loss(x, n, d, c, k, bias, 1.0, label, loss, stats, ws)
        vlq.vlq_softmax_loss_backward(x, n, d, c, k, bias, 1.0, label, stats, grad, dx, dc, db, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x2, c2, b2, l2, g2 = problem(F32, n, d, k, seed=turn + 1)
        for a, b in ((x, x2), (c, c2), (bias, b2), (label, l2), (grad, g2)):
            a.copy_(b)
        want = run(vlq, x, c, bias, 1.0, label, grad)
        for v in (loss, dx, dc, db):
            v.fill_(9.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for name, v in (("loss", loss), ("dx", dx), ("dc", dc), ("db", db)):
            assert torch.equal(v, want[name]), (turn, name)


def test_two_streams(vlq):
    a, b = problem(BF16, 500, 128, 3000, seed=1), problem(F16, 400, 96, 2000, seed=2)
    want = [run(vlq, v[0], v[1], v[2], 1.0, v[3], v[4]) for v in (a, b)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for s, v in ((s1, a), (s2, b)):
        with torch.cuda.stream(s):
            got.append(run(vlq, v[0], v[1], v[2], 1.0, v[3], v[4]))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for name in w:
            assert torch.equal(w[name], g[name]), name


def test_no_rows(vlq):
    x, c, bias, label, grad = problem(F32, 4, 8, 50)
    got = run(vlq, x[:0], c, bias, 1.0, label[:0], grad[:0])
    assert (got["dc"] == 0).all() and (got["db"] == 0).all()


def test_no_rows_many_centroids(vlq):
    # 2^32 values and more, each a thread's
    d, k = 257, 1 << 24
    x, c = torch.empty(0, d, dtype=BF16, device=DEV), torch.empty(k, d, dtype=BF16, device=DEV)
    got = run(vlq, x, c, None, 1.0, torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV), what=("dc",))
    assert (got["dc"][:1000] == 0).all() and (got["dc"][-1000:] == 0).all() and not got["dc"].any()
