"""vlq_clip_grads where a norm leaves fp32 and where a launch's table of tensors is full."""
import pytest
import torch

from test_gpu_clip_grads import BF16, DEV, F16, F32, check, clip, vlq  # noqa: F401

pytestmark = pytest.mark.gpu


def test_finite_norm_beyond_fp32(vlq):  # noqa: F811
    # 6e38: the values are clipped, and the norm says so by being finite
    top = torch.finfo(F32).max
    for t in (F32, BF16):
        grads = [torch.full((3,), 3e38, device=DEV).to(t), torch.tensor([-3e38], device=DEV)]
        want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
        outs, norm = clip(vlq, grads, 1e38)
        assert norm.item() == top
        limit = float(torch.tensor(1e38, dtype=F32))
        for g, o in zip(grads, outs):
            ref = g.double() * limit / want
            assert ((o.double() - ref).abs() <= ref.abs() * (torch.finfo(t).eps / 2 + 2.0 ** -22)).all()
        assert clip(vlq, grads, 1.0, out=False)[1].item() == top


@pytest.mark.parametrize("many", [139, 140, 141, 279, 280, 281])
def test_full_tables(vlq, many):  # noqa: F811
    # 140 tensors with values a launch; empty ones before, at and behind the boundary do not count among them
    g = torch.Generator().manual_seed(many)
    grads = [torch.randn(1 + 37 * i % 501, generator=g).to((F32, F16, BF16)[i % 3]).to(DEV) for i in range(many)]
    check(grads, *clip(vlq, grads, 1.0), 1.0)
    for at in (0, 138, 139, 140, 141, many):
        grads.insert(min(at, len(grads)), torch.empty(0, dtype=BF16, device=DEV))
    outs, norm = clip(vlq, grads, 1.0)
    check(grads, outs, norm, 1.0)
    kept = [v.clone() for v in grads]
    same, again = clip(vlq, kept, 1.0, in_place=True)
    assert torch.equal(norm, again) and all(torch.equal(a, b) for a, b in zip(outs, same))
