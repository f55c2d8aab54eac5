"""vlq_softmax_loss and its gradient where their range or their bits could end: probabilities whose terms cancel, in every form and
type, against the formulas in 64 bits."""

import pytest
import torch

from learn_reference import half_step, softmax_loss
from test_gpu_softmax_loss import BF16, F16, F32, DEV, run, vlq  # noqa: F401

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
