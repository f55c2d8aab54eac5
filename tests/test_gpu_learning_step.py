"""The operators together, as a program uses them: rows go to their nearest cells of an index, a transform per cell, back with
weights; a softmax loss over the cells; all gradients through to the inputs, clipped, and a step.  Against the same program in
64 bits with torch's differentiation, and captured into a graph."""
import math

import pytest
import torch

from learn_reference import U
from test_gpu_parity import CASES, dev, make_index
from util import problem

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def vlq():
    import paper_1901_00275_amd as vlq

    vlq.lib()
    return vlq


def cells_of(vlq, w):
    """Queries, their w nearest cells and the distances to them, from an index's own traversal."""
    kw, w1, w2, K = CASES["sift_ragged"]
    pr = problem(**kw)
    idx = make_index(vlq, pr, base=pr.X)
    nq = len(pr.Y)
    od, oi = torch.empty(nq, K, device=DEV), torch.empty(nq, K, dtype=torch.int32, device=DEV)
    cells, dist = torch.empty(nq, w, dtype=torch.int32, device=DEV), torch.empty(nq, w, device=DEV)
    vlq.vlq_search_debug(idx, dev(pr.Y), nq, w, min(w2, w), K, od, oi, cells, dist, None, None)
    torch.cuda.synchronize()
    vlq.vlq_index_free(idx)
    return dev(pr.Y), dev(pr.C), cells, dist


class Step:
    """One step: z = sum_c a_c (x o m_cell) (a scale per cell and component), loss = mean softmax loss of z against the centroids."""

    def __init__(self, vlq, x, C, cells, weight, scale):
        self.vlq, self.x, self.C, self.cells, self.weight, self.scale = vlq, x, C, cells, weight, scale
        (self.n, self.d), self.k, self.w = x.shape, C.shape[0], cells.shape[1]
        n, d, k, w = self.n, self.d, self.k, self.w
        new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
        self.m = torch.ones(k, d, device=DEV) + 0.01 * torch.arange(k, device=DEV)[:, None]
        self.label = cells[:, 0].contiguous()
        self.grad = torch.full((n,), 1.0 / n, device=DEV)
        self.off, self.place, self.source = new(k + 1, t=torch.int64), new(n, w, t=torch.int32), new(n * w, t=torch.int32)
        self.y, self.z, self.loss, self.stats = new(n * w, d), new(n, d), new(n), new(n, 2)
        self.dz, self.dC, self.dt, self.da, self.dx = new(n, d), new(k, d), new(n * w, d), new(n, w), new(n, d)
        self.norm, self.out = new(1), [new(k, d), new(n, w), new(n, d)]
        size = max(vlq.vlq_softmax_loss_workspace(torch.float32, n, d, k, b) for b in (0, 1))
        self.ws = new(size, t=torch.uint8)
        self.wg = new(vlq.vlq_group_rows_workspace(n, w, k), t=torch.uint8)
        self.wc = new(vlq.vlq_clip_grads_workspace(self.out), t=torch.uint8)

    def __call__(self):
        v, n, d, k, w = self.vlq, self.n, self.d, self.k, self.w
        v.vlq_group_rows(self.cells, n, w, k, self.off, self.place, self.source, self.wg)
        v.vlq_gather_rows(self.x, n, w, d, self.source, self.y)
        # the cell of every place: the work per cell (here a product by component) runs on contiguous rows
        cell = self.cells.reshape(-1)[self.source.long()].long()
        t = self.y * self.m[cell]
        v.vlq_combine_rows(t, n, w, d, self.place, self.weight, self.z)
        v.vlq_softmax_loss(self.z, n, d, self.C, k, None, self.scale, self.label, self.loss, self.stats, self.ws)
        v.vlq_softmax_loss_backward(self.z, n, d, self.C, k, None, self.scale, self.label, self.stats, self.grad, self.dz, self.dC, None, self.ws)
        v.vlq_combine_rows_backward(self.dz, t, n, w, d, self.place, self.weight, self.dt, self.da)
        dy = self.dt * self.m[cell]
        v.vlq_combine_rows(dy, n, w, d, self.place, None, self.dx)
        v.vlq_clip_grads([self.dC, self.da, self.dx], 0.5, self.out, self.norm, self.wc)
        return [self.loss, self.norm, *self.out]


def make(vlq):
    x, C, cells, dist = cells_of(vlq, 4)
    unit = float(C.norm(dim=1).mean())
    x, C = (x / unit).contiguous(), (C / unit).contiguous()
    weight = torch.softmax(-dist / unit ** 2, 1).contiguous()
    return Step(vlq, x, C, cells, weight, 8.0)


def test_step_against_64_bits(vlq):
    s = make(vlq)
    loss, norm, *out = s()
    x, C, a = (v.double().requires_grad_() for v in (s.x, s.C, s.weight))
    z = (a[:, :, None] * x[:, None, :] * s.m.double()[s.cells.long()]).sum(1)
    l = s.scale * (z @ C.t())
    want = torch.logsumexp(l, 1) - l.gather(1, s.label.long()[:, None])[:, 0]
    want.mean().backward()
    # Errors of an fp32 program in norms: the logits are off by (d / 4 + 80) U of their terms' sizes, and z by some 10 U of
    # its own; every gradient is p - [j = y] (off by twice the logits' error) times operands that are off by less
    mass = s.scale * float((z.detach().abs() @ C.detach().abs().t()).max())
    dl = mass * (s.d / 4 + 80) * U + 20 * U * mass
    assert float((loss.double() - want.detach()).abs().max()) <= 2 * dl + 512 * U
    grads = [C.grad, a.grad, x.grad]
    total = math.sqrt(sum(float((g ** 2).sum()) for g in grads))
    by = min(1.0, 0.5 / total)
    # a row's share: |p error| sums to at most 4 dl over the centroids, times the largest operand
    rows = 4 * dl + 1024 * U
    big = {0: float(z.detach().abs().max()), 1: float(C.detach().abs().max()) * float((x.detach().abs() * s.m.max()).sum(1).max()), 2: float(C.detach().abs().max() * s.m.max())}
    slack = 0.0
    for i, (g, o) in enumerate(zip(grads, out)):
        tol = rows * s.scale * big[i] * (1.0 if i == 0 else 1.0 / s.n)
        slack = max(slack, tol * math.sqrt(g.numel()))
        assert float((o.double() - g * by).abs().max()) <= tol + 2 * tol * math.sqrt(sum(v.numel() for v in grads)) / total * float(g.abs().max()) * by
    assert abs(norm.item() - total) <= 3 * slack + 4 * U * total


def test_step_captured_and_replayed(vlq):
    s = make(vlq)
    s()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = s()
    for turn in range(3):
        s.x.mul_(1.0 + 0.1 * turn)
        want = [v.clone() for v in s()]
        torch.cuda.synchronize()
        for v in res:
            v.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, res):
            assert torch.equal(a, b), turn


def test_steps_in_a_row(vlq):
    """A short descent runs: every step's gradients are finite and the clipped norm stays inside its bound."""
    s = make(vlq)
    for _ in range(5):
        loss, norm, dC, da, dx = s()
        assert torch.isfinite(loss).all() and math.isfinite(norm.item())
        assert math.sqrt(sum(float((v.double() ** 2).sum()) for v in (dC, da, dx))) <= 0.5 * (1 + 8 * U) + 1e-6
        s.C -= 0.1 * dC


def test_codebook_softened_by_the_recipe(vlq):
    """One gradient step of the training recipe moves the centroids as the 64-bit loss says; the recipe runs with such steps."""
    from datagen import codebooks

    g = torch.Generator().manual_seed(3)
    X = torch.randn(3000, 32, generator=g).to(DEV)
    Cb = X[:64].clone()
    vlq.vlq_kmeans(X, 3000, 32, 64, 5, Cb)
    before = Cb.clone()
    codebooks.soften_cells(vlq, X, Cb, 1, batch=3000, rate=0.1, max_norm=1e9)
    C = before.double().requires_grad_()
    d2 = ((X.double()[:, None, :] - C[None]) ** 2).sum(2)
    near = d2.detach().min(1)
    v = near.values.mean()
    (torch.logsumexp(-d2 / (2 * v), 1) - (-d2 / (2 * v)).gather(1, near.indices[:, None])[:, 0]).mean().backward()
    # step = rate v gradient: v to fp32 (3 000 sums of 32 squares: some 100 U), logits of <x, c> / v and the bias off by (D / 4 + 80) U
    # of sizes up to |x||c| / v, the gradient's two halves up to |x| and |c| / v in size, the centroid itself by U
    size = float(X.norm(dim=1).max() * before.norm(dim=1).max() / v)
    tol = 0.1 * float(X.abs().max() + before.abs().max()) * (4 * size * 88 * U + 600 * U) + 2 * U * float(before.abs().max())
    assert float((Cb.double() - (before.double() - 0.1 * v * C.grad)).abs().max()) <= tol
    C2, P = codebooks.train_with_library(vlq, X, 64, 4, 4, iters=2, soft_steps=3)
    assert torch.isfinite(C2).all() and torch.isfinite(P).all()


def test_two_steps_at_once(vlq):
    # on two streams, each with buffers of its own
    steps = [make(vlq) for _ in range(2)]
    steps[1].x.mul_(1.25)
    want = [[v.clone() for v in step()] for step in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        for step in steps:
            for v in (step.loss, step.norm, *step.out):
                v.fill_(9.0)
        torch.cuda.synchronize()
        for stream, step in zip(streams, steps):
            with torch.cuda.stream(stream):
                step()
        torch.cuda.synchronize()
        for step, ref in zip(steps, want):
            for a, b in zip((step.loss, step.norm, *step.out), ref):
                assert torch.equal(a, b)
