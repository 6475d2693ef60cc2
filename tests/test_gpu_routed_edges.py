"""Widths and values of the operators round the grouped products where their arithmetic or their launches have an edge, against their formulas in
64 bits.  Needs an MI355X."""
import pytest
import torch

import routed_reference as ref
import test_gpu_routed_ops as ops
from paper_2212_01185_amd import binding
from test_gpu_routed_ops import BF16, FP16, FP32
from train_reference import assert_near

pytestmark = pytest.mark.gpu


# weights and sums that fill 64 KB of LDS but for a kernel's own variables, on both sides; shapes whose last lanes have no eight
@pytest.mark.parametrize("features", [4080, 4088, 4095, 8176, 8184, 8191, 10000, 12301])
def test_layer_norm_of_widths_whose_weights_fill_64_kb(features):
    for i, (x_type, y_type) in enumerate(((BF16, BF16), (FP32, FP32), (FP32, FP16))):
        pad = (0, 3, 5)[i]
        x, gamma, beta, dy, off = ops._norm_inputs(x_type, y_type, features, [3, 0, 2], 1, features + i, pad)
        ops._check_norm(x, gamma, beta, dy, off, y_type, 1, pad=pad, what=(x_type, y_type))


# rows from the smallest that an eps of 2^-126 tells from 0 to those whose squares are just numbers, with gradients to both sides of theirs
@pytest.mark.parametrize("size,dsize,eps", [(1e-20, 100.0, 2.0 ** -126), (1e-12, 1e-8, 1e-30), (1.0, 1e25, 1e-5), (1.0, 1e-25, 1e-5), (1e12, 1e3, 1e-5), (1e17, 1e-8, 1e-5), (1e17, 1e8, 1.0)])
@pytest.mark.parametrize("features", [8, 36, 160, 513, 2056, 4096, 8193, 16384, 20000])
def test_layer_norm_gradient_of_rows_of_any_size(features, size, dsize, eps):
    gen = torch.Generator().manual_seed(features)
    for x_type, y_type in ((FP32, FP32), (FP32, BF16)):
        x = size * (torch.randn(6, features, generator=gen) + 0.5)
        dy = (dsize * torch.randn(6, features, generator=gen)).to(y_type)
        gamma = 1 + 0.3 * torch.randn(1, features, generator=gen)
        mean = x.double().mean(1, keepdim=True)
        stats = torch.cat([mean, (x.double().var(1, keepdim=True, correction=0) + eps) ** -0.5], 1).float()
        got = binding.pcc_layer_norm_grad(dy.cuda(), x.cuda(), stats.cuda(), gamma.cuda())
        for name, t, (value, limit) in zip(("dx", "dgamma", "dbeta"), got, ref.layer_norm_grad(dy, x, stats, gamma, [0, 6])):
            assert value.abs().max() < 1e38
            assert_near(t, value, limit, (name, x_type, y_type))
