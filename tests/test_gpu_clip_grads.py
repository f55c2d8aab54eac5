"""vlq_clip_grads against 64 bits: types mixed in one call, many tensors (several tables), odd sizes and alignment, in place,
empty tensors, values whose squares leave fp32, norms that are not finite."""
import math

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


def clip(vlq, grads, limit, in_place=False, out=True):
    outs = None if not out else grads if in_place else [torch.full_like(g, 7.0) for g in grads]
    norm = torch.full((1,), 7.0, device=DEV)
    ws = torch.full((vlq.vlq_clip_grads_workspace(grads),), 255, dtype=torch.uint8, device=DEV)
    vlq.vlq_clip_grads(grads, limit, outs, norm, ws)
    return outs, norm


def check(grads, outs, norm, limit):
    # fp64 sums of exact squares: the norm is rounded once to fp32; a value once more by the fp32 factor and product, and to its type
    want = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))
    assert abs(norm.item() - want) <= want * U * 1.01
    by = limit / want if want > limit else 1.0
    for g, o in zip(grads, outs):
        ref = g.double() * by
        tol = ref.abs() * (half_step(g.dtype) + 3 * U) + (2.0 ** -25 if g.dtype == F16 else 2.0 ** -133 if g.dtype == BF16 else 2.0 ** -149)
        assert ((o.double() - ref).abs() <= (tol if by < 1.0 else 0.0)).all()


@pytest.mark.parametrize("limit", [0.5, 1e9])
@pytest.mark.parametrize("counts", [[1], [7], [8192], [8193, 1, 0, 5], [100_001, 3, 70_000], [0, 0, 9], [1_000_003]])
@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_against_64_bits(vlq, t, counts, limit):
    g = torch.Generator().manual_seed(sum(counts))
    grads = [torch.randn(c, generator=g).to(t).to(DEV) for c in counts]
    outs, norm = clip(vlq, grads, limit)
    check(grads, outs, norm, limit)
    kept = [v.clone() for v in grads]
    same, norm2 = clip(vlq, kept, limit, in_place=True)
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(outs, same))
    _, norm3 = clip(vlq, grads, limit, out=False)
    assert torch.equal(norm, norm3)


@pytest.mark.parametrize("many", [79, 80, 81, 400])
def test_many_tensors_of_all_types(vlq, many):
    g = torch.Generator().manual_seed(many)
    grads = []
    for i in range(many):
        t = (F32, F16, BF16)[i % 3]
        v = torch.randn(int(torch.randint(0, 3000, (1,), generator=g)) + i % 5 + 2, generator=g).to(t).to(DEV)
        grads.append(v[1:] if i % 4 == 0 else v)  # (off 16 bytes)
    outs, norm = clip(vlq, grads, 1.0)
    check(grads, outs, norm, 1.0)


def test_more_parts_than_one_workgroup_adds(vlq):
    grads = [torch.randn(3, device=DEV) for _ in range(8300)]
    outs, norm = clip(vlq, grads, 2.0)
    check(grads, outs, norm, 2.0)


def test_large(vlq):
    g = torch.Generator(device=DEV).manual_seed(1)
    grads = [torch.randn(40_000_003, generator=g, device=DEV).to(BF16), torch.randn(5_000_001, generator=g, device=DEV)]
    outs, norm = clip(vlq, grads, 3.0)
    check(grads, outs, norm, 3.0)


@pytest.mark.parametrize("t", [F32, F16, BF16])
def test_unaligned(vlq, t):
    g = torch.Generator().manual_seed(9)
    for off in (1, 2, 3, 5):
        grads = [torch.randn(c + off, generator=g).to(t).to(DEV)[off:] for c in (1, 6, 20_001, 300_007)]
        outs = [torch.full((v.numel() + off - 1,), 7.0, dtype=t, device=DEV)[off - 1:] for v in grads]
        norm = torch.empty(1, device=DEV)
        vlq.vlq_clip_grads(grads, 0.5, outs, norm, torch.empty(vlq.vlq_clip_grads_workspace(grads), dtype=torch.uint8, device=DEV))
        check(grads, outs, norm, 0.5)


def test_larger_than_the_cache(vlq):
    g = torch.Generator(device=DEV).manual_seed(2)
    grads = [torch.randn(c, generator=g, device=DEV).to(t) for c, t in ((90_000_001, BF16), (30_000_007, F32), (50_000_003, F16))]
    outs, norm = clip(vlq, grads, 3.0)
    check(grads, outs, norm, 3.0)
    same, norm2 = clip(vlq, grads, 3.0, in_place=True)
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(outs, same))


def test_squares_beyond_fp32(vlq):
    for size in (1e30, 1e-30):
        grads = [torch.tensor([3.0, 4.0], device=DEV) * size]
        outs, norm = clip(vlq, grads, size)
        assert abs(norm.item() / (5 * size) - 1) < 1e-6
        check(grads, outs, norm, float(torch.tensor(size, dtype=F32)))


def test_factor_below_fp32(vlq):
    # 2^-300 of the norm: the values come out among the smallest of fp32, the factor is none of them
    grads = [torch.tensor([3.0, 4.0, 0.0], device=DEV) * 2.0 ** 125, torch.tensor([2.0], device=DEV, dtype=BF16)]
    for limit in (2.0 ** -100, 5 * 2.0 ** -140, 1e-3):
        outs, norm = clip(vlq, grads, limit)
        check(grads, outs, norm, limit)


def test_norm_that_is_not_finite(vlq):
    for bad in (math.inf, -math.inf, math.nan):
        grads = [torch.ones(100, device=DEV), torch.ones(50, device=DEV, dtype=BF16)]
        grads[1][7] = bad
        outs, norm = clip(vlq, grads, 0.1)
        assert not math.isfinite(norm.item())
        assert torch.equal(outs[0], grads[0]) and torch.equal(torch.nan_to_num(outs[1]), torch.nan_to_num(grads[1]))


def test_nothing(vlq):
    _, norm = clip(vlq, [], 1.0)
    assert norm.item() == 0.0
    outs, norm = clip(vlq, [torch.zeros(10, device=DEV)], 1.0)
    assert norm.item() == 0.0 and (outs[0] == 0).all()


def test_no_limit(vlq):
    grads = [torch.randn(1000, device=DEV)]
    outs, _ = clip(vlq, grads, math.inf)
    assert torch.equal(outs[0], grads[0])


def test_captured_and_replayed(vlq):
    grads = [torch.empty(c, device=DEV, dtype=t) for c, t in ((20_000, F32), (333, BF16), (9_999, F16))]
    outs = [torch.empty_like(g) for g in grads]
    norm = torch.empty(1, device=DEV)
    ws = torch.empty(vlq.vlq_clip_grads_workspace(grads), dtype=torch.uint8, device=DEV)
    for v in grads:
        v.normal_()
    vlq.vlq_clip_grads(grads, 1.0, outs, norm, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vlq.vlq_clip_grads(grads, 1.0, outs, norm, ws)
    for _ in range(4):
        for v in grads:
            v.normal_()
        want, wnorm = clip(vlq, grads, 1.0)
        for v in (*outs, norm):
            v.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, wnorm) and all(torch.equal(a, b) for a, b in zip(outs, want))
