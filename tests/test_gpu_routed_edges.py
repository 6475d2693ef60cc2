"""Widths and values of the operators round the grouped products where their arithmetic or their launches have an edge, against their formulas in
64 bits.  Needs an MI355X."""
import pytest
import torch

import test_gpu_routed_ops as ops
from test_gpu_routed_ops import BF16, FP16, FP32

pytestmark = pytest.mark.gpu


# weights and sums that fill 64 KB of LDS but for a kernel's own variables, on both sides; shapes whose last lanes have no eight
@pytest.mark.parametrize("features", [4080, 4088, 4095, 8176, 8184, 8191, 10000, 12301])
def test_layer_norm_of_widths_whose_weights_fill_64_kb(features):
    for i, (x_type, y_type) in enumerate(((BF16, BF16), (FP32, FP32), (FP32, FP16))):
        pad = (0, 3, 5)[i]
        x, gamma, beta, dy, off = ops._norm_inputs(x_type, y_type, features, [3, 0, 2], 1, features + i, pad)
        ops._check_norm(x, gamma, beta, dy, off, y_type, 1, pad=pad, what=(x_type, y_type))
