"""Plain 64-bit forms of the operators for learning cells by gradient, and how far a kernel's results may be from them.

A bound counts roundings: u(t) is half a step of a type relative to the value, U = 2^-24 that of fp32.  Products of fp16 or
bf16 values are exact in fp32; an fp32 value enters as two fp16 parts, off by 2^-23 of itself, and of the four products of two the
smallest (2^-22) is left out, so a product is off by 2^-21 = 8 U.  A sum of N products on the matrix cores is taken to round at
most N / 4 + 64 times (32 products an instruction, at most eight roundings in it).
"""
import torch

U = 2.0 ** -24
SUB = 2.0 ** -40  # what falls below the last bit of the two fp16 parts of a value, relative to the largest of its scale


def half_step(t):
    return torch.finfo(t).eps / 2


def softmax_loss(x, c, bias, scale, label, grad=None):
    """loss, dx, dc, dbias in 64 bits, and the bounds of the errors of each, from the same operands."""
    t = x.dtype
    n, d = x.shape
    k = c.shape[0]
    keep = (label >= 0) & (label < k)
    at = torch.where(keep, label, 0).long()[:, None]
    left = torch.ones(k, dtype=torch.bool, device=c.device) if bias is None else ~torch.isneginf(bias)
    X = torch.where(keep[:, None], x.double(), 0.0)
    Cc = torch.where(left[:, None], c.double(), 0.0)
    b = torch.zeros(k, dtype=torch.float64, device=c.device) if bias is None else bias.double()
    l = scale * (X @ Cc.t().contiguous()) + b
    some = bool(left.any())
    m = l.max(1, keepdim=True).values
    e = torch.exp(l - m) if some else torch.zeros_like(l)
    z = e.sum(1, keepdim=True)
    mine = l.gather(1, at)
    loss = torch.where(keep, (m - mine + torch.log(z))[:, 0], 0.0) if some else torch.where(keep, torch.inf, 0.0).double()
    # logits: products and their sum, the factor, the bias
    entry = 8 * U if t == torch.float32 else 0.0
    mass = abs(scale) * (X.abs() @ Cc.abs().t().contiguous())
    big = torch.where(torch.isneginf(l), 0.0, l.abs()).max(1, keepdim=True).values
    sub = abs(scale) * d * 2 * 2.0 ** -32 * X.abs().max(1, keepdim=True).values * Cc.abs().max() if t != torch.float16 else 0.0
    if t == torch.float32:
        sub = sub * 2.0 ** -8
    dl = (mass.max(1, keepdim=True).values * ((d / 4 + 64) * U + entry) + sub + 8 * U * big)
    dloss = torch.where(keep, (2 * dl + (k / 32 + 128) * U + 8 * U * (m.abs() + torch.where(torch.isneginf(mine), 0.0, mine).abs()))[:, 0], 0.0)
    out = {"loss": (loss, dloss), "m": m[:, 0], "z": z[:, 0]}
    if grad is None:
        return out
    g = torch.where(keep & torch.tensor(some, device=c.device), grad.double(), 0.0)[:, None]
    p = e / z if some else e
    P = p.clone()
    P.scatter_add_(1, at, torch.full_like(mine, -1.0))
    G = P * g
    # P: the exponent's error, the sum of the exponentials, two factors; its rounding to one or two fp16 parts; what is below those
    parts = 2.0 ** -22 if t == torch.float32 else 2.0 ** -11
    dP = p * (2 * dl + (k / 32 + 160) * U) + P.abs() * (parts + 8 * U) + SUB * (0.5 if t == torch.float32 else 1.0)
    low = (2.0 ** -40 if t == torch.float32 else 2.0 ** -32 if t == torch.bfloat16 else 0.0)
    top = g.abs().max() if n else 0.0
    dG = dP * g.abs() + SUB * top
    acc = lambda N: (N / 4 + 64) * U + entry + 8 * U  # noqa: E731
    dx = scale * (G @ Cc)
    bx = abs(scale) * ((dP * g.abs()) @ Cc.abs() + (G.abs() @ (Cc.abs() + 0.0)) * acc(k) + G.abs().sum(1, keepdim=True) * low * Cc.abs().max())
    dc = scale * (G.t().contiguous() @ X)
    bc = abs(scale) * (dG.t().contiguous() @ X.abs() + (G.abs().t().contiguous() @ X.abs()) * acc(n) + G.abs().sum(0)[:, None] * low * X.abs().max())
    db = G.sum(0)
    bb = (dP * g.abs()).sum(0) + G.abs().sum(0) * (n / 4 + 64) * U
    out["dx"] = (dx, bx + half_step(t) * (dx.abs() + bx) + 2.0 ** -149)
    out["dc"] = (dc, bc + half_step(t) * (dc.abs() + bc) + 2.0 ** -149)
    if t == torch.float16:  # the smallest steps of fp16
        out["dx"] = (dx, out["dx"][1] + 2.0 ** -25)
        out["dc"] = (dc, out["dc"][1] + 2.0 ** -25)
    out["db"] = (db, bb + 8 * U * db.abs())
    return out


def check(got, want, what):
    ref, tol = want
    got = got.double()
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin), f"{what}: finite in other places"
    assert torch.equal(got[~fin], ref[~fin]), f"{what}: infinities differ"
    off = torch.where(fin, (got - ref).abs() - tol, torch.zeros_like(tol))
    if off.numel():
        i = off.argmax()
        assert off.max() <= 0, (f"{what}: {got.reshape(-1)[i].item()!r} for {ref.reshape(-1)[i].item()!r}, bound "
                                f"{tol.expand_as(ref).reshape(-1)[i].item():.3g}, {(off > 0).sum().item()} of {off.numel()} outside")
