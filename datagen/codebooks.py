"""Seeded codebook training recipe run through the GPU library (inputs for the benchmark and the
full-size tests): seeded initial codebooks from the training sample, then every step by the
library's own calls.  This module holds no arithmetic of the method: it draws the initial rows and
sequences library calls (and puts the two gradients of a centroid together); the library module is passed in by the caller.
"""
from __future__ import annotations

import torch

from . import MASTER_SEED, STREAM_KMEANS, _gen


def _seeded_init(X: torch.Tensor, k: int, seed: int, stream: int) -> torch.Tensor:
    """An initial codebook for Lloyd iterations: k seeded rows of X (jittered copies if X has fewer rows)."""
    g = _gen("cpu", seed, STREAM_KMEANS, stream)
    nt = X.shape[0]
    if nt >= k:
        init = torch.randperm(nt, generator=g)[:k]
    else:
        init = torch.randint(0, nt, (k,), generator=g)
    Cb = X[init.to(X.device)].clone()
    if nt < k:
        Cb += 1e-3 * torch.randn(Cb.shape, generator=g).to(X.device) * (X.std() + 1e-6)
    return Cb.contiguous()


def soften_cells(vlq, X: torch.Tensor, Cb: torch.Tensor, steps: int, batch: int = 4096, rate: float = 0.1, max_norm: float = 1.0,
                 seed: int = MASTER_SEED):
    """Gradient steps of a trained first-level codebook Cb [k x D] (in place): the mean loss of a seeded batch's rows against
    their nearest centroids under the softmax over -||x - c||^2 / (2 v), v the batch's mean squared distance per cell.
    -||x - c||^2 / (2 v) is <x, c> / v - ||c||^2 / (2 v) up to a row's constant: a scale and a bias, whose gradient goes to
    the centroids as well.  The gradient is clipped to max_norm, in units of sqrt(v).  Returns the last batch's losses."""
    k, D = Cb.shape
    n = min(batch, X.shape[0])
    new = lambda *shape, **kw: torch.empty(*shape, device=X.device, **kw)  # noqa: E731
    assign, loss, stats, grad = new(n, dtype=torch.int32), new(n), new(n, 2), torch.full((n,), 1.0 / n, device=X.device)
    dC, dbias, clipped, norm = new(k, D), new(k), new(k, D), new(1)
    ws = new(max(vlq.vlq_softmax_loss_workspace(torch.float32, n, D, k, b) for b in (False, True)), dtype=torch.uint8)
    wc = new(vlq.vlq_clip_grads_workspace([dC]), dtype=torch.uint8)
    g = _gen("cpu", seed, STREAM_KMEANS, 1 << 20)
    for _ in range(steps):
        x = X[torch.randperm(X.shape[0], generator=g)[:n].to(X.device)].contiguous()
        vlq.vlq_kmeans(x, n, D, k, 0, Cb, assign)
        v = float(((x - Cb[assign.long()]) ** 2).sum(1).mean()) + 1e-20
        bias = -0.5 / v * (Cb * Cb).sum(1)
        vlq.vlq_softmax_loss(x, n, D, Cb, k, bias, 1.0 / v, assign, loss, stats, ws)
        vlq.vlq_softmax_loss_backward(x, n, D, Cb, k, bias, 1.0 / v, assign, stats, grad, None, dC, dbias, ws)
        dC -= dbias[:, None] * Cb / v
        dC *= v ** 0.5
        vlq.vlq_clip_grads([dC], max_norm, [clipped], norm, wc)
        Cb -= rate * v ** 0.5 * clipped
    return loss


def train_with_library(vlq, Xtrain: torch.Tensor, k: int, n: int, m: int, iters: int = 10, seed: int = MASTER_SEED,
                       pq_sample: int = 1 << 18, grid=(0.0, 0.0), soft_steps: int = 0):
    """Lloyd-trained C [k x D] and P [m x 256 x D/m], every step run by the GPU library: Lloyd iterations by
    vlq_kmeans (and on request soft_steps gradient steps behind them), the n-NN graph by vlq_build_index, line-quantisation
    residuals by vlq_line_residuals, and one 256-word codebook per sub-space by vlq_kmeans again."""
    nt, D = Xtrain.shape
    assert D % m == 0
    ds = D // m
    Cb = _seeded_init(Xtrain, k, seed, 0)
    vlq.vlq_kmeans(Xtrain, nt, D, k, iters, Cb)
    if soft_steps:
        soften_cells(vlq, Xtrain, Cb, soft_steps, seed=seed)
    # an index over the trained centroids (placeholder PQ codebooks) gives cells, lines and lambda bytes
    idx = vlq.vlq_build_index(vlq.vlq_params_t(D, k, n, m, grid[0], grid[1]), Cb, torch.zeros(m, 256, ds, device=Xtrain.device))
    try:
        ns = min(nt, pq_sample)
        R = torch.empty(ns, D, device=Xtrain.device)
        vlq.vlq_line_residuals(idx, Xtrain[:ns].contiguous(), ns, R)
    finally:
        vlq.vlq_index_free(idx)
    P = []
    for p in range(m):
        Rp = R[:, p * ds:(p + 1) * ds].contiguous()
        Pp = _seeded_init(Rp, 256, seed, 1 + p)
        vlq.vlq_kmeans(Rp, ns, ds, 256, iters, Pp)
        P.append(Pp)
    torch.cuda.synchronize()
    return Cb, torch.stack(P).contiguous()
