"""The operators for learning cells by gradient, as cases that can be timed and compared.

* ``loss``     softmax cross entropy of rows against all k centroids (or an output layer's k rows), the logits not kept;
* ``train``    the same with its gradient: loss, then the gradients of rows, centroids and bias;
* ``group``    rows sorted by the cells they were given to (the grouping and the gather);
* ``combine``  grouped rows back to their row's place, weighted and summed; ``combine_back`` its gradient;
* ``clip``     the global norm of many gradient tensors and their clipped values.

With ``own`` false ``run`` computes them in their plain form, elementary torch operations in 32 bits; with ``own`` true
through the library.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def listed():
    return [
        # one descriptor of an interactive user scored against the cells: latency
        dict(name="loss_1_fp32", do="loss", dtype="fp32", n=1, d=96, k=16_384, bias=True, scale=8.0, skip=0.0),
        # the output layer of one token, and of a small batch of an evaluation
        dict(name="loss_1_bf16", do="loss", dtype="bf16", n=1, d=1_024, k=65_536, bias=False, scale=1.0, skip=0.0),
        dict(name="loss_1000_fp16", do="loss", dtype="fp16", n=1_000, d=512, k=16_384, bias=True, scale=1.0, skip=0.05),
        # a training step of the cells of deep descriptors: small batch, then the largest codebook with an odd batch
        dict(name="train_cells_256", do="train", dtype="fp32", n=256, d=96, k=16_384, bias=True, scale=8.0, skip=0.0),
        dict(name="train_cells_4095", do="train", dtype="fp32", n=4_095, d=128, k=65_536, bias=True, scale=8.0, skip=0.02),
        # a training step of an output layer, rows of padding among its tokens, a vocabulary of odd size
        dict(name="train_output_bf16", do="train", dtype="bf16", n=8_192, d=2_048, k=50_001, bias=False, scale=1.0, skip=0.1),
        # a handful of requests routed to their cells
        dict(name="group_17", do="group", dtype="bf16", n=17, d=1_024, w=8, cells=64, drop=0.0),
        # all queries of a collection sorted by their probed cells
        dict(name="group_10000_cells", do="group", dtype="fp32", n=10_000, d=96, w=64, cells=65_536, drop=0.0),
        # a batch of tokens back from their experts, some pairs dropped, and the gradient of that
        dict(name="combine_16384", do="combine", dtype="bf16", n=16_384, d=2_048, w=8, cells=128, drop=0.03),
        dict(name="combine_back_5003", do="combine_back", dtype="bf16", n=5_003, d=1_024, w=6, cells=64, drop=0.03),
        # the gradients of a first-level codebook and of the product quantiser's codebooks
        dict(name="clip_codebooks", do="clip", dtype="fp32", tensors=9, values=2_129_920, limit=1.0),
        # the gradients of a model, many tensors of uneven size
        dict(name="clip_model_bf16", do="clip", dtype="bf16", tensors=291, values=400_000_000, limit=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["loss", "train", "train", "group", "combine", "combine_back", "clip"])
    dtype = rng.choice(["fp32", "fp16", "bf16"])
    if do in ("loss", "train"):
        n, d, k = _log(rng, 1, 8_192), _log(rng, 16, 2_048), _log(rng, 2, 65_536)
        while n * d * k > 8_192 * 2_048 * 50_001 // (4 if dtype == "fp32" else 1):
            n, d, k = _log(rng, 1, 8_192), _log(rng, 16, 2_048), _log(rng, 2, 65_536)
        if rng.random() < 0.6:
            d = max(16, d // 32 * 32)
        return dict(do=do, dtype=dtype, n=n, d=d, k=k, bias=rng.random() < 0.5, scale=rng.choice([1.0, 0.5, 8.0 if k >= 4_096 else 2.0]) if dtype == "fp32" else 1.0,
                    skip=rng.choice([0.0, 0.1]))
    if do == "clip":
        tensors = _log(rng, 1, 300)
        return dict(do=do, dtype=dtype, tensors=tensors, values=max(tensors, _log(rng, 1_000, 200_000_000)), limit=rng.choice([0.5, 1.0, 1e9]))
    n, d, w = _log(rng, 1, 16_384), _log(rng, 16, 2_048), rng.choice([1, 2, 4, 6, 8, 64])
    while n * w * d > 16_384 * 2_048 * 8:
        n, d, w = _log(rng, 1, 16_384), _log(rng, 16, 2_048), rng.choice([1, 2, 4, 6, 8, 64])
    if rng.random() < 0.6:
        d = max(16, d // 32 * 32)
    return dict(do=do, dtype=dtype, n=n, d=d, w=w, cells=max(w, _log(rng, 8, 65_536)), drop=rng.choice([0.0, 0.03]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _inputs(case, seed):
    """The inputs of a case in their own types, from the seed alone."""
    g = torch.Generator(device=DEV).manual_seed(1_000_003 * int(seed) + 17)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    uni = lambda *s: torch.rand(*s, generator=g, device=DEV)  # noqa: E731
    t = TYPES[case["dtype"]]
    do = case["do"]
    if do in ("loss", "train"):
        n, d, k = case["n"], case["d"], case["k"]
        # centroids of unit length; descriptors around the one they belong to, or (16-bit types) the last layer's rows, whose
        # logits spread by two units, with the right one among the larger ones
        c = torch.nn.functional.normalize(rnd(k, d), dim=1)
        label = torch.randint(0, k, (n,), generator=g, device=DEV, dtype=torch.int32)
        if case["dtype"] == "fp32":
            x = c[label.long()] + 0.7 * rnd(n, d) / math.sqrt(d)
        else:
            x = 0.6 * math.log(k) * c[label.long()] + 2.0 * rnd(n, d)
        label = torch.where(uni(n) < case["skip"], torch.full_like(label, -1), label)
        s = {"x": x.to(t), "c": c.to(t), "label": label, "bias": None, "grad": (0.5 + uni(n)) / n}
        if case["bias"]:
            # squared distances: -scale / 2 |x - c|^2 up to a row's constant; and a prior of the cells
            s["bias"] = -0.5 * case["scale"] * (s["c"].float() ** 2).sum(1) + 0.5 * rnd(k)
        return s
    if do == "clip":
        n, values = case["tensors"], case["values"]
        share = np.random.default_rng(n).uniform(0.02, 1.0, n) ** 3  # one layout for all seeds, as a model has
        counts = np.maximum(1, (share / share.sum() * (values - n)).astype(np.int64))
        return {"grads": [(rnd(int(v)) * 0.01).to(t) for v in counts]}
    n, d, w, cells = case["n"], case["d"], case["w"], case["cells"]
    if cells >= 4 * w:
        # w cells of every row, near ones more often: a start and different steps, popular cells first
        start = (uni(n, 1) ** 2 * cells).long()
        step = 1 + (uni(n, 1) * (cells // w - 1)).long()
        cell = ((start + step * torch.arange(w, device=DEV)) % cells).int()
    else:
        cell = torch.argsort(uni(n, cells), dim=1)[:, :w].int()
    if case["drop"]:
        cell = torch.where(uni(n, w) < case["drop"], torch.full_like(cell, -1), cell)
    s = {"cell": cell.contiguous()}
    if do == "group":
        s["x"] = rnd(n, d).to(t)
        return s
    s["weight"] = torch.softmax(rnd(n, w), dim=1)
    s["y"] = rnd(n * w, d).to(t)
    if do == "combine_back":
        s["dout"] = rnd(n, d).to(t)
    return s


def _places(cell):
    """(from, place) of the stable sort of the pairs by cell, dropped pairs (negative cells) behind all others."""
    flat = cell.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, 1 << 40), flat)
    order = torch.argsort(key, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    return torch.where(flat[order] < 0, -1, order).int(), torch.where(flat < 0, -1, place).int().view(cell.shape)


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    t = TYPES[case["dtype"]]
    # what a user's program keeps from call to call: buffers for the outputs and the workspace
    if case["do"] in ("loss", "train"):
        n, d, k = case["n"], case["d"], case["k"]
        s["loss"], s["stats"] = torch.empty(n, device=DEV), torch.empty(n, 2, device=DEV)
        if case["do"] == "train":
            s["dx"], s["dc"] = torch.empty(n, d, dtype=t, device=DEV), torch.empty(k, d, dtype=t, device=DEV)
            s["db"] = torch.empty(k, device=DEV) if case["bias"] else None
        if own:
            import paper_1901_00275_amd as vlq

            size = max(vlq.vlq_softmax_loss_workspace(t, n, d, k, b) for b in ((0, 1) if case["do"] == "train" else (0,)))
            s["ws"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    elif case["do"] == "clip":
        # the clipped gradients lie in one piece, each on a boundary of 256 bytes
        counts = [g.numel() for g in s["grads"]]
        size = 256 // BYTES[case["dtype"]]
        starts = np.cumsum([0] + [-(-v // size) * size for v in counts])
        s["whole"] = torch.zeros(int(starts[-1]), dtype=t, device=DEV)
        s["out"] = [s["whole"][int(a):int(a) + v] for a, v in zip(starts, counts)]
        s["norm"] = torch.empty(1, device=DEV)
        if own:
            import paper_1901_00275_amd as vlq

            s["ws"] = torch.empty(vlq.vlq_clip_grads_workspace(s["grads"]), dtype=torch.uint8, device=DEV)
    else:
        n, d, w = case["n"], case["d"], case["w"]
        if case["do"] == "group":
            s["off"] = torch.empty(case["cells"] + 1, dtype=torch.int64, device=DEV)
            s["place"] = torch.empty(n, w, dtype=torch.int32, device=DEV)
            s["source"] = torch.empty(n * w, dtype=torch.int32, device=DEV)
            s["y"] = torch.zeros(n * w, d, dtype=t, device=DEV)
            if own:
                import paper_1901_00275_amd as vlq

                s["ws"] = torch.empty(vlq.vlq_group_rows_workspace(n, w, case["cells"]), dtype=torch.uint8, device=DEV)
        else:
            s["place"] = _places(s["cell"])[1].contiguous()
            if case["do"] == "combine":
                s["out"] = torch.empty(n, d, dtype=t, device=DEV)
            else:
                s["dy"] = torch.zeros(n * w, d, dtype=t, device=DEV)
                s["dweight"] = torch.empty(n, w, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _run_own(s):
    import paper_1901_00275_amd as vlq

    do = s["do"]
    if do in ("loss", "train"):
        n, d, k = s["n"], s["d"], s["k"]
        vlq.vlq_softmax_loss(s["x"], n, d, s["c"], k, s["bias"], s["scale"], s["label"], s["loss"], s["stats"], s["ws"])
        if do == "loss":
            return {"loss": s["loss"]}
        vlq.vlq_softmax_loss_backward(s["x"], n, d, s["c"], k, s["bias"], s["scale"], s["label"], s["stats"], s["grad"],
                                      s["dx"], s["dc"], s["db"], s["ws"])
        return {"loss": s["loss"], "dx": s["dx"], "dc": s["dc"], "db": s["db"]}
    if do == "clip":
        vlq.vlq_clip_grads(s["grads"], s["limit"], s["out"], s["norm"], s["ws"])
        return {"norm": s["norm"], "out": s["whole"]}
    n, d, w = s["n"], s["d"], s["w"]
    if do == "group":
        vlq.vlq_group_rows(s["cell"], n, w, s["cells"], s["off"], s["place"], s["source"], s["ws"])
        vlq.vlq_gather_rows(s["x"], n, w, d, s["source"], s["y"])
        return {"off": s["off"], "place": s["place"], "source": s["source"], "y": s["y"]}
    if do == "combine":
        vlq.vlq_combine_rows(s["y"], n, w, d, s["place"], s["weight"], s["out"])
        return {"out": s["out"]}
    vlq.vlq_combine_rows_backward(s["dout"], s["y"], n, w, d, s["place"], s["weight"], s["dy"], s["dweight"])
    return {"dy": s["dy"], "dweight": s["dweight"]}


def run(s):
    if own:
        return _run_own(s)
    do, t = s["do"], TYPES[s["dtype"]]
    if do in ("loss", "train"):
        x, c, keep = s["x"].float(), s["c"].float(), s["label"] >= 0
        at = s["label"].long().clamp(min=0)[:, None]
        logits = (x @ c.t()) * s["scale"]
        if s["bias"] is not None:
            logits = logits + s["bias"]
        m = logits.max(1, keepdim=True).values
        mine = logits.gather(1, at)
        e = torch.exp(logits - m)
        z = e.sum(1, keepdim=True)
        loss = torch.where(keep, (m - mine + torch.log(z))[:, 0], 0.0)
        if do == "loss":
            return {"loss": loss}
        g = torch.where(keep, s["grad"], 0.0)[:, None]
        p = e / z
        p.scatter_add_(1, at, torch.full_like(mine, -1.0))
        p = p * g
        return {"loss": loss, "dx": ((p @ c) * s["scale"]).to(t), "dc": ((p.t() @ x) * s["scale"]).to(t),
                "db": p.sum(0) if s["bias"] is not None else None}
    if do == "clip":
        norm = torch.stack([(g.float() ** 2).sum() for g in s["grads"]]).sum().sqrt()
        by = torch.clamp(s["limit"] / norm, max=1.0)
        _ = [o.copy_(g.float() * by) for o, g in zip(s["out"], s["grads"])]
        return {"norm": norm[None], "out": s["whole"]}
    n, d, w = s["n"], s["d"], s["w"]
    if do == "group":
        source, place = _places(s["cell"])
        count = torch.zeros(s["cells"] + 1, dtype=torch.int64, device=DEV)
        flat = s["cell"].reshape(-1).long()
        count.index_add_(0, flat + 1, (flat >= 0).long())
        count[0] = 0
        row = torch.div(source.clamp(min=0), w, rounding_mode="floor").long()
        y = torch.where((source >= 0)[:, None], s["x"][row], 0)
        return {"off": count.cumsum(0), "place": place, "source": source, "y": y}
    place, there = s["place"].long().clamp(min=0), s["place"] >= 0
    weight = torch.where(there, s["weight"], 0.0)
    y = s["y"][place].float()  # [n, w, d]
    if do == "combine":
        return {"out": (y * weight[:, :, None]).sum(1).to(t)}
    dout = s["dout"].float()
    dweight = torch.where(there, (y * dout[:, None, :]).sum(2), 0.0)
    # pairs without a place are sent to a row behind the last one, which is cut off
    dy = torch.zeros(n * w + 1, d, dtype=t, device=DEV)
    dy[torch.where(there, place, n * w).reshape(-1)] = (weight[:, :, None] * dout[:, None, :]).to(t).reshape(n * w, d)
    return {"dy": dy[: n * w], "dweight": dweight}


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    e, do = BYTES[case["dtype"]], case["do"]
    if do in ("loss", "train"):
        n, d, k = case["n"], case["d"], case["k"]
        read = (n + k) * d * e + 4 * n + (4 * k if case["bias"] else 0)
        if do == "loss":
            return {"bytes": read + 4 * n, "flops": 2.0 * n * d * k}
        return {"bytes": read + 4 * n + 4 * n + (n + k) * d * e + (4 * k if case["bias"] else 0), "flops": 6.0 * n * d * k}
    if do == "clip":
        return {"bytes": 2.0 * case["values"] * e, "flops": 3.0 * case["values"]}
    n, d, w = case["n"], case["d"], case["w"]
    pairs = n * w * (1 - case["drop"])
    if do == "group":
        return {"bytes": 4 * n * w + 8 * n * w + 8 * (case["cells"] + 1) + (n + pairs) * d * e, "flops": n * w}
    if do == "combine":
        return {"bytes": 8 * n * w + (pairs + n) * d * e, "flops": 2.0 * pairs * d}
    return {"bytes": 8 * n * w + 4 * n * w + (2 * pairs + n) * d * e, "flops": 3.0 * pairs * d}


def exact(case, seed):
    """By the definitions, in 64 bits: the loss by log-sum-exp and its gradient through torch's differentiation in blocks of rows;
    the grouping by lists on the host; the sums row by row over the choices."""
    s, do = _inputs(case, seed), case["do"]
    if do in ("loss", "train"):
        n, d, k = case["n"], case["d"], case["k"]
        if n * d * k > 2e12:
            return None
        c = s["c"].double().requires_grad_(do == "train")
        b = None if s["bias"] is None else s["bias"].double().requires_grad_(do == "train")
        loss, dx = [], []
        rows = max(1, min(n, (1 << 27) // k))
        for i in range(0, n, rows):
            x = s["x"][i:i + rows].double().requires_grad_(do == "train")
            y = s["label"][i:i + rows].long()
            dots = torch.mm(x, c.transpose(0, 1).contiguous())
            logits = dots * case["scale"] if b is None else dots * case["scale"] + b[None, :]
            term = torch.logsumexp(logits, 1) - logits[torch.arange(y.numel(), device=DEV), y.clamp(min=0)]
            term = torch.where(y < 0, torch.zeros_like(term), term)
            loss.append(term.detach())
            if do == "train":
                (term * s["grad"][i:i + rows].double()).sum().backward()
                dx.append(x.grad)
        if do == "loss":
            return {"loss": torch.cat(loss)}
        return {"loss": torch.cat(loss), "dx": torch.cat(dx), "dc": c.grad, "db": None if b is None else b.grad}
    if do == "clip":
        norm = math.sqrt(math.fsum(float((g.double() * g.double()).sum()) for g in s["grads"]))
        by = case["limit"] / norm if norm > case["limit"] else 1.0
        size = 256 // BYTES[case["dtype"]]
        pad = lambda v: torch.nn.functional.pad(v, (0, -v.numel() % size))  # noqa: E731
        return {"norm": np.array([norm]), "out": torch.cat([pad(g.double() * by) for g in s["grads"]])}
    n, d, w = case["n"], case["d"], case["w"]
    flat = s["cell"].cpu().numpy().reshape(-1)
    order = np.lexsort((np.arange(n * w), np.where(flat < 0, np.int64(1) << 40, flat)))
    at = np.full(n * w, -1, np.int64)
    at[order] = np.arange(n * w)
    at[flat < 0] = -1
    if do == "group":
        row = torch.from_numpy(np.where(flat[order] < 0, -1, order // w)).to(DEV)
        y = torch.zeros(n * w, d, dtype=torch.float64, device=DEV)
        y[row >= 0] = s["x"][row[row >= 0]].double()
        return {"off": None, "place": None, "source": None, "y": y}
    at = torch.from_numpy(at.reshape(n, w)).to(DEV)
    out = torch.zeros(n, d, dtype=torch.float64, device=DEV)
    dy = torch.zeros(n * w, d, dtype=torch.float64, device=DEV) if do == "combine_back" else None
    dweight = torch.zeros(n, w, dtype=torch.float64, device=DEV)
    for j in range(w):
        rows = torch.nonzero(at[:, j] >= 0)[:, 0]
        y = s["y"][at[rows, j]].double()
        a = s["weight"][rows, j].double()[:, None]
        if do == "combine":
            out[rows] += a * y
        else:
            dout = s["dout"][rows].double()
            dy[at[rows, j]] = a * dout
            dweight[rows, j] = (dout * y).sum(1)
    return {"out": out} if do == "combine" else {"dy": dy, "dweight": dweight}
