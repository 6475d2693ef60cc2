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


SHAPES = [5, 8, 30, 120, 160, 240, 513, 960, 1000, 2056, 3000, 4096, 8193, 12301, 16384, 20000, 40001, 65536]


@pytest.mark.parametrize("features", SHAPES)
def test_layer_norm_of_rows_of_one_value_is_beta(features):
    """Whatever the value, the mean is it: no distance, and a width of the root of eps."""
    gen = torch.Generator().manual_seed(features)
    wild = (1 + torch.rand(40, generator=gen)) * 10.0 ** torch.randint(-18, 19, (40,), generator=gen) * (torch.randint(0, 2, (40,), generator=gen) * 2 - 1)
    values = torch.cat([torch.tensor([0.0, 1.0, -3.0, 12032.0, 12345.678, 1e-20, 1e15, 0.1, 1e30]), wild])
    gamma, beta = torch.randn(1, features, generator=gen).cuda(), torch.randn(1, features, generator=gen).cuda()
    for dtype, eps in ((BF16, 1e-5), (FP16, 1e-5), (FP32, 1e-5), (FP32, 1e-30)):
        x = values.to(dtype)
        x = x[torch.isfinite(x)][:, None].expand(-1, features).contiguous().cuda()
        y, stats = binding.pcc_layer_norm(x, gamma, beta, eps=eps, out_dtype=dtype)
        assert torch.equal(stats[:, 0], x[:, 0].float())
        assert ((stats[:, 1].double() * eps ** 0.5 - 1).abs() <= 4 * ref.U).all()      # eps in fp32 (a half), 1 / sqrt of the hardware (one step)
        assert torch.equal(y, beta.to(dtype).expand(len(x), -1))


def _norm_bounds(x, gamma, beta, eps):
    """y, the statistics and their bounds where a mean may be far from 0 against the width: the mean is right but for its own rounding and those of
    the sum of the distances from a first mean, which is off by a sum's roundings."""
    x = x.double().cpu()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = (d * d).mean(1, keepdim=True)
    s = (var + eps) ** -0.5
    h = d * s
    away = d.abs().mean(1, keepdim=True)
    first = (ref.DEPTH + 2) * ref.U * x.abs().mean(1, keepdim=True)
    # a wave's mean and the row's are rounded to fp32; distances from the first mean are as large as d and its error
    e_mean = 2 * ref.U * mean.abs() + (ref.DEPTH + 4) * ref.U * (away + first)
    # squares about the first mean, of which what its error adds is taken off: 1/64 of them at most, else they are summed anew
    e_var = (ref.DEPTH + 8) * ref.U * var * (1 + 1 / 32) + 2 * away * e_mean + e_mean ** 2
    low = (var + eps - e_var).clamp_min(eps / 2)
    e_s = s * (e_var / (2 * low) + 5 * ref.U)
    e_h = s * e_mean + 3 * ref.U * h.abs() + (d.abs() + e_mean) * e_s
    g, b = gamma.double().cpu(), beta.double().cpu()
    return (g * h + b, g.abs() * e_h + 2 * ref.U * ((g * h + b).abs() + (g * h).abs())), (torch.cat([mean, s], 1), torch.cat([e_mean, e_s], 1))


@pytest.mark.parametrize("features", SHAPES)
def test_layer_norm_of_rows_far_from_0(features):
    """Means of up to a million widths, and rows with one value that is far larger than all others, first, last or between."""
    gen = torch.Generator().manual_seed(features + 1)
    x = torch.randn(40, features, generator=gen)
    x[:20] = x[:20] * 10.0 ** torch.linspace(-6, 0, 20)[:, None] + torch.randn(20, 1, generator=gen) + 1
    for i, at in enumerate((0, features - 1, features // 2)):
        x[20 + i, at], x[24 + i, at] = 1e4, -1e7
    gamma, beta = torch.randn(1, features, generator=gen), torch.randn(1, features, generator=gen)
    for eps in (1e-5, 1e-14):
        y, stats = binding.pcc_layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), eps=eps)
        (want, bound), (want_stats, stats_bound) = _norm_bounds(x, gamma, beta, eps)
        assert_near(stats, want_stats, stats_bound, ("stats", eps))
        assert_near(y, want, bound, ("y", eps))
    # a row's bits do not hang on its neighbours
    alone = torch.cat([binding.pcc_layer_norm(x[i:i + 1].cuda(), gamma.cuda(), beta.cuda(), eps=1e-14)[0] for i in range(40)])
    assert torch.equal(alone, y)


@pytest.mark.parametrize("experts,k", [(3, 2), (8, 2), (12, 2), (64, 8), (65, 3), (200, 16), (1000, 4)])
@pytest.mark.parametrize("dtype", [FP32, BF16, FP16])
def test_route_gradient_of_a_masked_logit_is_0_beside_what_is_not_a_number(dtype, experts, k):
    """Experts that may not be taken keep a gradient of 0 where the token's other gradients are NaN or infinite."""
    gen = torch.Generator().manual_seed(experts)
    logits = torch.randn(70, experts, generator=gen)
    dweight = torch.randn(70, k, generator=gen)
    logits[::7, 0], logits[1::7, 0] = float("nan"), float("inf")
    dweight[2::7, 0], dweight[3::7, 1], dweight[4::7, 0] = float("nan"), float("inf"), -float("inf")
    plain = torch.zeros(70, dtype=torch.bool)
    plain[5::7] = plain[6::7] = True
    logits[:, experts // 2::2] = -float("inf")
    logits = logits.to(dtype)
    masked = logits == -float("inf")
    for over_all in (False, True):
        expert, weight = binding.pcc_route(logits.cuda(), k, over_all=over_all)
        got = binding.pcc_route_grad(dweight.cuda(), logits.cuda(), expert, weight, over_all=over_all).cpu()
        assert (got[masked] == 0).all()
        if over_all:                                # each open one's gradient hangs on all of them: p (0 - sum w dw) at least is not finite
            assert not torch.isfinite(got[~plain][~masked[~plain]]).any()
        value, limit = ref.route_grad(torch.where(expert.cpu() >= 0, dweight, torch.zeros(())), logits, expert.cpu(), k, over_all)
        assert_near(got[plain], value[plain], limit[plain], (dtype, over_all))


@pytest.mark.parametrize("k", [-1, 0, 17, 1 << 50])
def test_route_refuses_a_number_of_choices_before_it_makes_room_for_them(k):
    with pytest.raises(binding.PccError):
        binding.pcc_route(torch.zeros(4, 32, device="cuda"), k)


@pytest.mark.parametrize("features", [8, 160, 4096, 16384, 20000])
def test_layer_norm_of_finite_rows_whose_squares_are_not(features):
    x = torch.full((3, features), 1e25)
    x[:, ::2] *= -1
    x[1] = 1e25 * (torch.randn(features, generator=torch.Generator().manual_seed(2)) + 3)
    beta = torch.randn(1, features, generator=torch.Generator().manual_seed(1)).cuda()
    for dtype in (FP32, BF16):
        y, stats = binding.pcc_layer_norm(x.to(dtype).cuda(), None, beta, out_dtype=dtype)
        assert (stats[:, 1] == 0).all() and torch.isfinite(stats).all() and torch.equal(y, beta.to(dtype).expand(3, -1))
