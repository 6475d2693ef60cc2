"""Layer norm, routing, rows by expert and dropout against their formulas in 64 bits.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import routed_reference as ref
from paper_2212_01185_amd import binding
from train_reference import assert_near

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [(BF16, BF16), (FP16, FP16), (FP32, FP32), (FP32, BF16), (FP32, FP16)]


def _wide(t, pad, fill=float("nan")):
    """The same matrix with its rows further apart, not at the start of an allocation."""
    if not pad:
        return t.cuda()
    full = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype)
    full[:, 1:1 + t.shape[1]] = t
    return full.cuda()[:, 1:1 + t.shape[1]]


def _offsets(lengths):
    return [0] + np.cumsum(lengths).tolist()


# ---------------------------------------------------------------------------------------------------- layer norm

# one feature, odd ones, the codec's widths, each number of lanes and eights that a row may have, to both sides of each border
FEATURES = [1, 2, 7, 30, 36, 64, 65, 128, 160, 191, 192, 193, 256, 257, 500, 512, 513, 1024, 1100, 2048, 2056, 4096, 4099, 8192, 8193, 16384]
HUGE = [16385, 32768, 40001, 65536]
LENGTHS = [([1], 0), ([0, 3, 0, 70, 1], 4), ([65, 64], 0), ([0, 0], 2)]


def _norm_inputs(x_type, y_type, features, lengths, tail, seed, pad=0):
    gen = torch.Generator().manual_seed(seed)
    rows, groups = sum(lengths) + tail, len(lengths)
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = ((normal(rows, features) + normal(features)) * torch.exp(normal(rows, 1)) + normal(rows, 1)).to(x_type)
    dy = normal(rows, features).to(y_type)
    if tail:                                        # what belongs to no group is not looked at
        x[-tail:], dy[-tail:] = float("nan"), float("inf")
    return _wide(x, pad), (1 + 0.5 * normal(groups, features)).cuda(), normal(groups, features).cuda(), _wide(dy, pad), torch.tensor(_offsets(lengths)).cuda()


def _check_norm(x, gamma, beta, dy, off, y_type, tail, eps=1e-5, pad=0, what=""):
    rows, features = x.shape
    y_full = torch.full((rows, features + pad), 5.0, dtype=y_type, device="cuda")
    stats = torch.full((rows, 2), 5.0, device="cuda")
    offsets = off.tolist() if off is not None else [0, rows]
    y, got_stats = binding.pcc_layer_norm(x, gamma, beta, off, eps=eps, out=y_full[:, :features], stats=stats)
    (want, bound), (want_stats, stats_bound) = ref.layer_norm(x, gamma, beta, offsets, eps)
    assert_near(y, want, bound, ("y", what))
    assert_near(got_stats, want_stats, stats_bound, ("stats", what))
    dx_full = torch.full((rows, features + pad), 5.0, dtype=x.dtype, device="cuda")
    dx, dgamma, dbeta = binding.pcc_layer_norm_grad(dy, x, stats, gamma, off, dx=dx_full[:, :features])
    for name, got, (value, limit) in zip(("dx", "dgamma", "dbeta"), (dx, dgamma, dbeta), ref.layer_norm_grad(dy, x, stats, gamma, offsets)):
        assert_near(got, value, limit, (name, what))
    if tail:
        assert (y[-tail:] == 5).all() and (stats[-tail:] == 5).all() and (dx[-tail:] == 5).all()
    assert (y_full[:, features:] == 5).all() and (dx_full[:, features:] == 5).all()


@pytest.mark.parametrize("lengths,tail", LENGTHS)
@pytest.mark.parametrize("features", FEATURES)
def test_layer_norm(features, lengths, tail):
    for i, (x_type, y_type) in enumerate(TYPES):
        pad = (0, 3, 8, 2, 0)[i]
        x, gamma, beta, dy, off = _norm_inputs(x_type, y_type, features, lengths, tail, features * 100 + len(lengths), pad)
        _check_norm(x, gamma, beta, dy, off, y_type, tail, pad=pad, what=(x_type, y_type))


@pytest.mark.parametrize("features", HUGE)
def test_layer_norm_of_the_widest_rows(features):
    for x_type, y_type, pad in ((BF16, BF16, 0), (FP32, FP16, 5)):
        x, gamma, beta, dy, off = _norm_inputs(x_type, y_type, features, [2, 0, 3], 1, features, pad)
        _check_norm(x, gamma, beta, dy, off, y_type, 1, pad=pad, what=(x_type, y_type))


@pytest.mark.parametrize("features,rows,groups", [(160, 30011, 1), (160, 20000, 5), (36, 50000, 3), (4096, 700, 2), (1000, 3000, 70), (24, 9000, 300)])
def test_layer_norm_of_many_rows(features, rows, groups):
    """Sums over chunks that are joined: values, and the same bits every time."""
    share = np.random.default_rng(rows).dirichlet(np.ones(groups))
    lengths = np.floor(share * rows).astype(int)
    lengths[0] += rows - lengths.sum()
    x, gamma, beta, dy, off = _norm_inputs(BF16, BF16, features, lengths.tolist(), 0, rows)
    _check_norm(x, gamma, beta, dy, off, BF16, 0)
    _, stats = binding.pcc_layer_norm(x, gamma, beta, off)
    first = binding.pcc_layer_norm_grad(dy, x, stats, gamma, off)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, binding.pcc_layer_norm_grad(dy, x, stats, gamma, off)))


def test_layer_norm_without_weights_or_offsets():
    x, gamma, beta, dy, off = _norm_inputs(BF16, BF16, 100, [300], 0, 1)
    for g, b in ((None, None), (gamma, None), (None, beta)):
        _check_norm(x, g, b, dy, None, BF16, 0)
        with_offsets, stats = binding.pcc_layer_norm(x, g, b, off)
        without, again = binding.pcc_layer_norm(x, g, b)
        assert torch.equal(with_offsets, without) and torch.equal(stats, again)
    y, none = binding.pcc_layer_norm(x, want_stats=False)
    assert none is None and torch.equal(y, binding.pcc_layer_norm(x)[0])
    dx, dgamma, dbeta = binding.pcc_layer_norm_grad(dy, x, stats, gamma)
    only, a, b = binding.pcc_layer_norm_grad(dy, x, stats, gamma, want_weights=False)
    assert a is None and b is None and torch.equal(only, dx)
    nothing, a, b = binding.pcc_layer_norm_grad(dy, x, stats, gamma, want_dx=False)
    assert nothing is None and torch.equal(a, dgamma) and torch.equal(b, dbeta)
    for i in range(2):                              # no rows: no result, and sums of nothing
        empty = x[:0]
        assert binding.pcc_layer_norm(empty, gamma, beta)[0].shape == (0, 100)
        _, a, b = binding.pcc_layer_norm_grad(empty, empty, stats[:0], gamma, None if i else torch.tensor([0, 0]).cuda())
        assert (a == 0).all() and (b == 0).all()


@pytest.mark.parametrize("features", [5, 160, 4096, 20000])
def test_layer_norm_of_rows_that_hardly_vary(features):
    """Equal values (a variance of 0 but for the mean's rounding), a mean far from 0 against the spread, very large and very small values."""
    gen = torch.Generator().manual_seed(features)
    rows = [torch.full((features,), v) for v in (0.0, 1.0, -3.0, 1e-20, 1e15)]
    rows += [1000 + 0.01 * torch.randn(features, generator=gen), 1e-18 * torch.randn(features, generator=gen), 1e15 * torch.randn(features, generator=gen)]
    x = torch.stack(rows).cuda()
    dy = torch.randn(x.shape, generator=gen).cuda()
    for eps in (1e-5, 1e-30, 1.0):
        y, stats = binding.pcc_layer_norm(x, eps=eps)
        (want, bound), (want_stats, stats_bound) = ref.layer_norm(x, None, None, [0, len(rows)], eps)
        e_mean = stats_bound[:, 0]
        assert ((stats[:, 0].double().cpu() - want_stats[:, 0]).abs() <= e_mean * 1.001 + 1e-44).all()
        # a rounded mean leaves distances of its error where there are none: |h| is at most sqrt(features) in any case
        flat = want_stats[:, 1] * e_mean > 0.1
        assert_near(y[~flat], want[~flat], bound[~flat], eps)
        assert torch.isfinite(y).all() and (y.abs() <= 1.01 * features ** 0.5).all()
        for got, (value, limit) in zip(binding.pcc_layer_norm_grad(dy[~flat], x[~flat], stats[~flat].contiguous())[:1],
                                       ref.layer_norm_grad(dy[~flat], x[~flat], stats[~flat], None, [0, int((~flat).sum())])):
            assert_near(got, value, limit, "dx")


def test_layer_norm_keeps_nan_and_infinity_in_their_rows():
    x, gamma, beta, dy, off = _norm_inputs(BF16, BF16, 160, [70, 60], 0, 4)
    x[5, 7], x[100, 0] = float("nan"), float("inf")
    y, stats = binding.pcc_layer_norm(x, gamma, beta, off)
    bad = torch.isnan(y).any(1)
    assert bad[5] and bad[100] and int(bad.sum()) == 2 and torch.isnan(y[5]).all()
    x[5, 7], x[100, 0] = 0, 0
    dy[90, 3] = float("nan")
    _, stats = binding.pcc_layer_norm(x, gamma, beta, off)
    dx, dgamma, dbeta = binding.pcc_layer_norm_grad(dy, x, stats, gamma, off)
    assert torch.isnan(dx[90]).all() and int(torch.isnan(dx).any(1).sum()) == 1
    assert int(torch.isnan(dgamma).sum()) == 1 and torch.isnan(dgamma[1, 3]) and int(torch.isnan(dbeta).sum()) == 1


def test_layer_norm_gradient_against_differences():
    """sum(c y) a small step along a direction of x, gamma and beta and against it, by the formula in 64 bits."""
    x, gamma, beta, dy, off = _norm_inputs(FP32, FP32, 40, [20, 0, 10], 0, 5)
    _, stats = binding.pcc_layer_norm(x, gamma, beta, off)
    grads = binding.pcc_layer_norm_grad(dy, x, stats, gamma, off)
    gen = torch.Generator().manual_seed(6)
    at = [t.double().cpu() for t in (x, gamma, beta)]
    c = dy.double().cpu()
    for i in range(3):
        e = torch.randn(at[i].shape, generator=gen, dtype=torch.float64)

        def value(step):
            moved = [t + step * e if j == i else t for j, t in enumerate(at)]
            return (c * ref.layer_norm(*moved, off.tolist(), 1e-5)[0][0]).sum().item()

        h = 1e-5
        slope = (value(h) - value(-h)) / (2 * h)
        parts = grads[i].double().cpu() * e
        # differences: h^2 of the third derivative (of the size of the gradient, rows have widths of 0.1 and more: 1e3), fp32 in the gradient
        assert abs(parts.sum().item() - slope) <= 1e-5 * parts.abs().sum().item() + 1e-6 * c.abs().sum().item()


def test_layer_norm_offsets_that_make_no_sense_stay_inside():
    x, gamma, beta, dy, _ = _norm_inputs(BF16, BF16, 48, [100, 100], 0, 3)
    for bad in ([0, 150, 90], [-5, 300, 1 << 40], [1 << 60, -(1 << 60), 7]):
        off = torch.tensor(bad).cuda()
        y, dx = (torch.full((220, 48), 5.0, dtype=BF16, device="cuda") for _ in range(2))
        stats = torch.full((220, 2), 5.0, device="cuda")
        binding.pcc_layer_norm(x, gamma, beta, off, out=y[10:210], stats=stats[10:210])
        binding.pcc_layer_norm_grad(dy, x, stats[10:210], gamma, off, dx=dx[10:210])
        torch.cuda.synchronize()
        for t in (y, dx, stats):
            assert (t[:10] == 5).all() and (t[210:] == 5).all()


def test_layer_norm_falling_offsets_stay_in_the_workspace():
    rows, groups, features = 60000, 20, 48
    x = torch.ones(rows, features, dtype=BF16, device="cuda")
    off = torch.tensor([0, rows] * 10 + [0]).cuda()
    need = binding.load().pcc_layer_norm_grad_workspace_bytes(rows, groups, features)
    space = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device="cuda")
    binding.pcc_layer_norm_grad(x, x, torch.ones(rows, 2, device="cuda"), None, off, workspace=space[:need])
    torch.cuda.synchronize()
    assert need > 0 and (space[need:] == 77).all()


# ---------------------------------------------------------------------------------------------------- routing

EXPERTS = [(1, 1), (2, 1), (3, 3), (8, 2), (9, 4), (16, 16), (17, 2), (32, 1), (60, 5), (64, 8), (65, 3), (128, 8), (200, 16), (256, 2), (500, 4), (512, 7), (1000, 16), (1024, 1)]


@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("experts,k", EXPERTS)
def test_route(experts, k, over_all):
    gen = torch.Generator().manual_seed(experts * 20 + k)
    for dtype, tokens, pad in ((FP32, 67, 0), (BF16, 130, 3), (FP16, 1, 2), (FP32, 9, 5)):
        logits = (3 * torch.randn(tokens, experts, generator=gen)).to(dtype)
        if tokens > 60:
            logits[3] = 1.5                          # ties: the lowest first
            logits[4] = -float("inf")                # none may be taken
            logits[5, 1:] = -float("inf")            # one may
            logits[6, ::2] = -float("inf")
            logits[7] = torch.finfo(dtype).min       # the lowest number is one
            logits[8] = torch.linspace(-80, 80, experts).to(dtype)
            logits[9] = 0.0
            logits[9, experts // 2:] = -0.0
        dweight = torch.randn(tokens, k, generator=gen)
        dweight[::3, 0] = 0
        l = _wide(logits, pad)
        expert, weight = binding.pcc_route(l, k, over_all=over_all)
        want, (w, bound) = ref.route(l, k, over_all)
        assert torch.equal(expert.cpu(), want)
        assert_near(weight, w, bound, (dtype, over_all))
        assert ((expert.cpu() >= 0) | (weight.cpu() == 0)).all()
        full = torch.full((tokens, experts + pad), 5.0, dtype=dtype, device="cuda")
        if tokens > 60:
            dweight[4] = float("nan")                # of choices that are none
        got = binding.pcc_route_grad(dweight.cuda(), l, expert, weight, over_all=over_all, dlogits=full[:, :experts])
        dweight = torch.where(want >= 0, dweight, torch.zeros(()))
        value, limit = ref.route_grad(dweight, l, want, k, over_all)
        assert_near(got, value, limit, ("gradient", dtype, over_all))
        assert (full[:, experts:] == 5).all() and (got[l == -float("inf")] == 0).all()


@pytest.mark.parametrize("dtype", [FP32, BF16, FP16])
def test_route_zeros_of_both_signs_are_equal(dtype):
    l = torch.zeros(3, 9, dtype=dtype)
    l[0, ::2], l[1, :5], l[2, 4:] = -0.0, -0.0, -0.0
    expert, weight = binding.pcc_route(l.cuda(), 4)
    assert expert.tolist() == [[0, 1, 2, 3]] * 3 and (weight == 0.25).all()


def test_route_nan_and_infinity():
    l = torch.zeros(4, 12)
    l[0, 7], l[1, 3], l[1, 9], l[2, 5] = float("nan"), float("inf"), -float("nan"), float("inf")
    for over_all in (False, True):
        expert, weight = binding.pcc_route(l.cuda(), 2, over_all=over_all)
        want, _ = ref.route(l, 2, over_all)
        assert torch.equal(expert.cpu(), want) and expert[:3, 0].tolist() == [7, 9, 5] and expert[1, 1] == 3
        assert torch.isnan(weight[:3]).any(1).all() and not torch.isnan(weight[3]).any()
        d = binding.pcc_route_grad(torch.ones(4, 2, device="cuda"), l.cuda(), expert, weight, over_all=over_all)
        assert torch.isnan(d[:3]).any(1).all() and torch.isfinite(d[3]).all()


def test_route_gradient_against_differences():
    gen = torch.Generator().manual_seed(3)
    l = torch.randn(20, 11, generator=gen)
    e, c = torch.randn(20, 11, generator=gen, dtype=torch.float64), torch.randn(20, 3, generator=gen)
    for over_all in (False, True):
        expert, weight = binding.pcc_route(l.cuda(), 3, over_all=over_all)
        got = binding.pcc_route_grad(c.cuda(), l.cuda(), expert, weight, over_all=over_all).double().cpu()
        h = 1e-6                                     # far less than two logits are apart: the choice stays
        up, down = (ref.route(l.double() + s * e, 3, over_all) for s in (h, -h))
        assert torch.equal(up[0], expert.cpu()) and torch.equal(down[0], expert.cpu())
        slope = ((up[1][0] - down[1][0]) * c.double()).sum().item() / (2 * h)
        assert abs((got * e).sum().item() - slope) <= 1e-5 * (got * e).abs().sum().item() + 1e-8


# ---------------------------------------------------------------------------------------------------- rows by expert

@pytest.mark.parametrize("tokens,k,experts", [(1, 1, 1), (1, 4, 8), (63, 2, 8), (64, 1, 3), (65, 3, 64), (500, 8, 256), (1000, 1, 1000), (4096, 1, 5), (4097, 1, 5), (3000, 2, 1024),
                                              (9000, 2, 16), (40000, 3, 7), (300000, 2, 64), (70001, 16, 1000)])
def test_expert_sort(tokens, k, experts):
    gen = np.random.default_rng(tokens + experts)
    for kind in range(3):
        if kind == 0:
            expert = gen.integers(0, experts, (tokens, k))
        elif kind == 1:                              # most to one, some to none, some numbers that no expert has
            expert = np.where(gen.random((tokens, k)) < 0.9, experts // 2, gen.integers(-2, experts + 3, (tokens, k)))
            expert[0, 0] = np.iinfo(np.int32).min
            expert[-1, -1] = np.iinfo(np.int32).max
        else:
            expert = np.full((tokens, k), -1)
        expert = torch.from_numpy(expert.astype(np.int32))
        offsets, place = binding.pcc_expert_sort(expert.cuda(), experts)
        key = expert.view(-1).long()
        there = (key >= 0) & (key < experts)
        order = torch.sort(torch.where(there, key, torch.full_like(key, experts)), stable=True).indices[:int(there.sum())]
        want = torch.full((tokens * k,), -1, dtype=torch.int32)
        want[order] = torch.arange(len(order), dtype=torch.int32)
        assert torch.equal(place.cpu().view(-1), want)
        assert torch.equal(offsets.cpu(), torch.cat([torch.zeros(1, dtype=torch.int64), torch.bincount(key[there], minlength=experts).cumsum(0)]))
        if tokens <= 500:
            slow = ref.sort(expert, experts)
            assert torch.equal(slow[0], offsets.cpu()) and torch.equal(slow[1], place.cpu())


def test_expert_sort_of_nothing():
    offsets, place = binding.pcc_expert_sort(torch.zeros(0, 2, dtype=torch.int32, device="cuda"), 5)
    assert offsets.tolist() == [0] * 6 and place.shape == (0, 2)


SHAPES = [(1, 1, 1, 8), (5, 2, 4, 1), (33, 2, 8, 30), (64, 1, 3, 7), (70, 4, 16, 160), (129, 8, 64, 36), (40, 3, 5, 1000), (9, 16, 20, 2056), (3, 2, 4, 65536), (1000, 2, 7, 128), (200, 5, 9, 513)]


@pytest.mark.parametrize("tokens,k,experts,features", SHAPES)
def test_rows_and_join(tokens, k, experts, features):
    gen = torch.Generator().manual_seed(tokens * 7 + features)
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    for i, (z_type, y_type) in enumerate(((BF16, BF16), (FP16, FP32), (FP32, FP32), (BF16, FP32), (FP16, FP16))):
        pad = (0, 3, 1, 8, 2)[i]
        expert = torch.randint(-1 if i % 2 else 0, experts, (tokens, k), generator=gen, dtype=torch.int32).cuda()
        offsets, place = binding.pcc_expert_sort(expert, experts)
        used, at = int(offsets[-1]), place.cpu().long()
        # rows
        x = _wide(normal(tokens, features).to(z_type), pad)
        full = torch.full((tokens * k + 2, features + pad), 5.0, dtype=z_type, device="cuda")
        rows = binding.pcc_expert_rows(x, place, out=full[:, :features])
        want = torch.full((tokens * k + 2, features + pad), 5.0, dtype=z_type)
        for j in range(k):
            want[at[at[:, j] >= 0, j], :features] = x.cpu()[at[:, j] >= 0]
        assert torch.equal(full.cpu(), want)
        # join, with weights and without
        z = normal(tokens * k, features).to(z_type)
        z[used:] = float("nan")                      # what is nobody's is not looked at
        z = _wide(z, pad)
        weight = normal(tokens, k).cuda()
        weight[0, 0] = 0
        for w in (weight, None):
            out = torch.full((tokens, features + pad), 5.0, dtype=y_type, device="cuda")
            y = binding.pcc_expert_join(z, place, w, out=out[:, :features])
            assert_near(y, *ref.join(z, place, w, tokens * k), ("join", z_type, y_type))
            assert (out[:, features:] == 5).all()
            dy = _wide(normal(tokens, features).to(y_type), pad)
            dz_full = torch.full((tokens * k, features + pad), 5.0, dtype=z_type, device="cuda")
            dz, dweight = binding.pcc_expert_join_grad(dy, z, place, w, dz=dz_full[:, :features])
            (want_dz, dz_bound), (want_dw, dw_bound) = ref.join_grad(dy, z, place, w, tokens * k)
            assert_near(dz, want_dz, dz_bound, ("dz", z_type, y_type))
            assert_near(dweight, want_dw, dw_bound, ("dweight", z_type, y_type))
            assert (dz_full[:, features:] == 5).all() and (dz[used:] == 5).all() and (dweight[place < 0] == 0).all()
            alone, none = binding.pcc_expert_join_grad(dy, z, place, w, want_dweight=False)
            assert none is None and torch.equal(alone[:used], dz[:used])


def test_places_outside_the_rows_are_left_out():
    """Places that no row has (of another sort, of a longer buffer): nothing is read or written there."""
    place = torch.tensor([[0, 7], [-1, 1 << 30], [3, -(1 << 31)], [9, 10]], dtype=torch.int32, device="cuda")
    x, z = torch.randn(4, 40, device="cuda"), torch.randn(10, 40, device="cuda")
    full = torch.full((30, 40), 5.0, device="cuda")
    binding.pcc_expert_rows(x, place, out=full[10:20])
    inside = full[10:20]
    assert torch.equal(inside[[0, 7, 3, 9]], x[[0, 0, 2, 3]]) and (full[:10] == 5).all() and (full[20:] == 5).all()
    assert (inside[[1, 2, 4, 5, 6, 8]] == 5).all()
    assert_near(binding.pcc_expert_join(z, place), *ref.join(z, place, None, 10), "join")
    assert (binding.pcc_expert_join(z, place)[1] == 0).all()
    _, dweight = binding.pcc_expert_join_grad(x, z, place)
    assert (dweight[[1, 1, 2, 3], [0, 1, 1, 1]] == 0).all()
    assert (binding.pcc_expert_join(z[:0], place) == 0).all()
    assert binding.pcc_expert_join(z, place[:0]).shape == (0, 40)


# ---------------------------------------------------------------------------------------------------- dropout

@pytest.mark.parametrize("rows,features", [(1, 1), (1, 8), (3, 7), (70, 30), (64, 64), (33, 160), (5, 1000), (2, 65536), (300, 9)])
def test_dropout(rows, features):
    gen = torch.Generator().manual_seed(rows * 11 + features)
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    seed, step = 0x0123456789ABCDEF, (7 << 32) + 5
    bits = ref.drop_bits(range(rows), features, seed, step)
    d_step = torch.tensor([step]).cuda()
    for i, (x_type, y_type) in enumerate(((BF16, BF16), (FP16, FP16), (FP32, FP32), (BF16, FP32), (FP32, BF16), (FP16, FP32), (FP32, FP16))):
        pad = (0, 3, 1, 8, 2, 0, 5)[i]
        x, residual = _wide(normal(rows, features).to(x_type), pad), _wide(normal(rows, features).to(y_type), pad)
        for p, r in ((0.0, None), (0.1, residual), (0.5, None), (1.0, residual), (0.999999, None), (1.0, None), (3e-6, residual)):
            full = torch.full((rows, features + pad), 5.0, dtype=y_type, device="cuda")
            y = binding.pcc_dropout(x, p, seed, step=d_step, residual=r, out=full[:, :features])
            assert_near(y, *ref.dropout(x, p, r, bits), (x_type, y_type, p))
            assert (full[:, features:] == 5).all()
            if r is None:                            # kept or 0, exactly
                border = int(p * 65536 + 0.5)
                assert torch.equal(y.cpu() == 0, (bits < border) | (x.cpu() == 0))


def test_dropout_masks():
    """The share that is kept, and that another seed, step, row or column has another mask."""
    rows, features, p = 2000, 1000, 0.3
    x = torch.ones(rows, features, device="cuda")
    kept = lambda **kw: binding.pcc_dropout(x, p, **dict(dict(seed=5, step=torch.tensor([1]).cuda()), **kw)) != 0  # noqa: E731
    first = kept()
    share = 1 - round(p * 65536) / 65536
    assert abs(first.double().mean().item() - share) <= 6 * (share * (1 - share) / (rows * features)) ** 0.5
    assert torch.equal(first, kept())
    same = share ** 2 + (1 - share) ** 2            # what two independent masks have in common
    for other in (kept(seed=6), kept(seed=5 + (1 << 32)), kept(step=torch.tensor([2]).cuda()), kept(step=torch.tensor([1 + (1 << 32)]).cuda()),
                  first.roll(1, 0), first.roll(1, 1), first.roll(8, 1)):
        assert abs((first == other).double().mean().item() - same) <= 6 * (same * (1 - same) / (rows * features)) ** 0.5
    assert torch.equal(kept(step=None), kept(step=torch.tensor([0]).cuda()))


def test_dropout_in_place_and_of_what_is_not_a_number():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(100, 36, generator=gen).to(BF16).cuda()
    r = torch.randn(100, 36, generator=gen).to(BF16).cuda()
    want = binding.pcc_dropout(x, 0.4, 9, residual=r)
    a, b = x.clone(), r.clone()
    assert torch.equal(binding.pcc_dropout(a, 0.4, 9, residual=r, out=a), want) and torch.equal(binding.pcc_dropout(x, 0.4, 9, residual=b, out=b), want)
    wild = torch.full((100, 36), float("nan"), dtype=BF16, device="cuda")
    wild[::2] = float("inf")
    y = binding.pcc_dropout(wild, 0.4, 9, residual=r)
    kept = binding.pcc_dropout(torch.ones_like(x), 0.4, 9) != 0
    assert torch.equal(y[~kept], r[~kept]) and not torch.isfinite(y[kept]).any()
    # the backward pass: the same mask on the gradient
    dy = torch.randn(100, 36, generator=gen).cuda()
    dx = binding.pcc_dropout(dy, 0.4, 9, out_dtype=BF16)
    assert torch.equal(dx != 0, kept)
