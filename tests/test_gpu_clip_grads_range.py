"""vlq_clip_grads where a norm leaves fp32."""
import pytest
import torch

from test_gpu_clip_grads import BF16, DEV, F32, clip, vlq  # noqa: F401

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
