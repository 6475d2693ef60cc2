"""The code length and its gradient where means lie far beyond every level.  Needs an MI355X."""
import math

import pytest
import torch

import train_reference as ref
from paper_2212_01185_amd import binding
from test_gpu_train_ops import TERM             # how far a term may be off, derived there

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dist", [0, 1])
@pytest.mark.parametrize("k", [3, 5, 7])
def test_loss_of_means_far_beyond_any_level(k, dist):
    """A component that is nowhere near has no share and no gradient, however far off it is: there are no infinities and no NaN."""
    gen = torch.Generator().manual_seed(10 * k + dist)
    far = [1e6, 1e18, 1e30, 1e36, 3e38, float("inf")]
    count = 2 * len(far) * 3
    params = torch.cat([torch.randn(count, 9 * k, generator=gen), 0.1 * torch.randn(count, 3 * k, generator=gen)], 1)
    level = torch.tensor([0, 255, 100]).repeat(count // 3)
    rgb = level[:, None].repeat(1, 3).to(torch.uint8)
    for c in range(3):
        params[:, 3 * k * c + k] = torch.tensor([s * v for v in far for s in (1, -1)]).repeat_interleave(3)
        params[:, 3 * k * c + 2 * k:3 * k * c + 3 * k] = 2 * torch.randn(count, k, generator=gen) - 4
    bits, grad = binding.pcc_mixture_loss(params.cuda(), rgb.cuda(), dist)
    finite = torch.where(torch.isinf(params), params.sign() * 3e38, params)
    want, size = ref.loss_gradient(finite, rgb, k, dist, 1.0)
    want_bits = ref.code_length(finite, rgb, k, dist)
    assert torch.isfinite(grad).all() and torch.isfinite(bits).all()
    assert ((grad.double().cpu() - want).abs() <= TERM * size + 2.0 ** -24 * want.abs() + 1e-12).all()
    assert ((bits.double().cpu() - want_bits).abs() <= 3 * (TERM / math.log(2) + 16 * 2.0 ** -23)).all()
