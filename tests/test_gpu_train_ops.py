"""The operators of a training step against their formulas in 64 bits.  Needs an MI355X."""
import math

import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2212_01185_amd import binding, synth

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def _offsets(lengths):
    return [0] + np.cumsum(lengths).tolist()


# ---------------------------------------------------------------------------------------------------- contexts

@pytest.mark.parametrize("nbhd,delay", [(10, 2), (12, 3), (12, 1)])
@pytest.mark.parametrize("n,h,w,width,ld", [(1, 1, 1, 40, 40), (2, 1, 5, 40, 40), (1, 6, 1, 36, 36), (1, 2, 2, 37, 41), (3, 7, 9, 40, 48), (1, 16, 33, 40, 40),
                                            (1, 5, 600, 40, 64), (2, 3, 259, 36, 36)])
def test_contexts(nbhd, delay, n, h, w, width, ld):
    img = np.random.default_rng(n * h * w).integers(0, 256, (n, h, w, 3), dtype=np.uint8)
    full = torch.full((n * h * w, ld), 7.0, dtype=BF16, device="cuda")
    out = binding.pcc_contexts(torch.from_numpy(img).cuda(), nbhd, delay, width, out=full[:, :width])
    want = torch.from_numpy(ref.contexts(img, nbhd, delay))
    got = full.double().cpu()
    assert torch.equal(got[:, :3 * nbhd], want) and out.data_ptr() == full.data_ptr()
    assert (got[:, 3 * nbhd:width] == 0).all() and (got[:, width:] == 7).all()


def test_contexts_are_what_the_oracle_gathers(orc, orc_diagonal, orc_paper):
    img = np.random.default_rng(1).integers(0, 256, (1, 5, 8, 3), dtype=np.uint8)
    for oracle, nbhd, delay in ((orc, 10, 2), (orc_paper, 12, 3), (orc_diagonal, 12, 1)):
        got = binding.pcc_contexts(torch.from_numpy(img).cuda(), nbhd, delay)
        assert got.shape[1] == -(-3 * nbhd // 8) * 8
        want = np.stack([oracle.gather(img[0], r, c) for r in range(5) for c in range(8)])
        assert np.array_equal(got[:, :3 * nbhd].double().cpu().numpy(), want)


# ---------------------------------------------------------------------------------------------------- grouped products

# (in, out): the codec's layers, odd ones, more than a tile
SHAPES = [(32, 160), (160, 160), (160, 128), (128, 60), (40, 128), (128, 36), (128, 84), (192, 192), (64, 64), (1, 1), (7, 13), (30, 33),
          (130, 257), (520, 136), (320, 520), (256, 520), (2, 300), (264, 40), (250, 6)]
# rows of the groups, and rows of no group behind them
GROUPS = [([1], 0), ([0, 3, 0, 130, 1], 5), ([127, 129], 0), ([0, 0], 3), ([333], 1)]


def _inputs(dtype, fan_in, fan_out, lengths, tail, act, seed, pad=0):
    gen = torch.Generator().manual_seed(seed)
    rows = sum(lengths) + tail
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = ref.activate(normal(rows, fan_in), act).to(dtype)
    w = (normal(len(lengths), fan_out, fan_in) / math.sqrt(fan_in)).to(dtype)
    dz = normal(rows, fan_out).to(dtype)
    bias = normal(len(lengths), fan_out)
    if tail:                                        # what belongs to no group is not looked at
        x[-tail:], dz[-tail:] = float("nan"), float("inf")

    def wide(t):                                    # rows further apart than they are long, and not at the start of an allocation
        if not pad:
            return t.cuda()
        full = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype)
        full[:, 1:1 + t.shape[1]] = t
        return full.cuda()[:, 1:1 + t.shape[1]]

    return wide(x), w.cuda(), bias.cuda(), wide(dz), torch.tensor(_offsets(lengths)).cuda()


@pytest.mark.parametrize("lengths,tail", GROUPS)
@pytest.mark.parametrize("fan_in,fan_out", SHAPES)
def test_grouped_linear(fan_in, fan_out, lengths, tail):
    seed = fan_in * 1000 + fan_out + len(lengths)
    for dtype, act, out_dtype, pad, with_bias in ((BF16, ref.RELU, BF16, 0, True), (FP16, ref.LEAKY, FP32, 3, True), (BF16, ref.NONE, FP32, 8, False),
                                                  (FP16, ref.RELU, FP16, 2, True)):
        x, w, bias, _, off = _inputs(dtype, fan_in, fan_out, lengths, tail, ref.NONE, seed, pad)
        out = torch.full((x.shape[0], fan_out + pad), 5.0, dtype=out_dtype, device="cuda")
        got = binding.pcc_grouped_linear(x, w, bias if with_bias else None, off, act, out=out[:, :fan_out])
        want, bound = ref.linear(x, w, bias if with_bias else None, off.tolist(), act)
        ref.assert_near(got, want, bound, (dtype, act, out_dtype))
        if tail:
            assert (got[-tail:] == 5).all()
        assert (out[:, fan_out:] == 5).all()


@pytest.mark.parametrize("lengths,tail", GROUPS)
@pytest.mark.parametrize("fan_in,fan_out", SHAPES)
def test_grouped_linear_grad(fan_in, fan_out, lengths, tail):
    seed = fan_in * 1000 + fan_out + len(lengths)
    for dtype, act, pad in ((BF16, ref.RELU, 0), (FP16, ref.LEAKY, 3), (BF16, ref.NONE, 8), (FP16, ref.RELU, 2)):
        x, w, _, dz, off = _inputs(dtype, fan_in, fan_out, lengths, tail, act, seed, pad)
        full = torch.full((x.shape[0], fan_in + pad), 5.0, dtype=dtype, device="cuda")
        dx, dw, db = binding.pcc_grouped_linear_grad(dz, x, w, off, act, dx=full[:, :fan_in])
        want = ref.linear_grad(dz, x, w, off.tolist(), act)
        for name, got, (value, bound) in zip(("dx", "dw", "db"), (dx, dw, db), want):
            ref.assert_near(got, value, bound, (name, dtype, act))
        if tail:
            assert (dx[-tail:] == 5).all()
        assert (full[:, fan_in:] == 5).all()
        none, dw2, db2 = binding.pcc_grouped_linear_grad(dz, x, w, off, act, want_dx=False)
        assert none is None and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("fan_in,fan_out,rows,groups", [(160, 160, 70001, 1), (128, 36, 40000, 3), (36, 128, 33333, 7), (64, 64, 20000, 40), (200, 520, 9000, 2),
                                                        (300, 264, 20000, 1), (17, 9, 30000, 2), (264, 1000, 17000, 2)])
def test_many_rows(fan_in, fan_out, rows, groups):
    """Sums over chunks that are joined: values, the same bits every time, and every group its own."""
    share = np.random.default_rng(rows).dirichlet(np.ones(groups))
    lengths = np.floor(share * rows).astype(int)
    lengths[0] += rows - lengths.sum()
    x, w, bias, dz, off = _inputs(BF16, fan_in, fan_out, lengths.tolist(), 0, ref.RELU, rows)
    y = binding.pcc_grouped_linear(x, w, bias, off, ref.RELU)
    want, bound = ref.linear(x, w, bias, off.tolist(), ref.RELU)
    ref.assert_near(y, want, bound, "y")
    first = binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU)
    for name, got, (value, bound) in zip(("dx", "dw", "db"), first, ref.linear_grad(dz, x, w, off.tolist(), ref.RELU)):
        ref.assert_near(got, value, bound, name)
    for _ in range(3):
        again = binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_gradient_of_a_product_against_differences():
    """The directional derivative of sum(c * y) for a layer behind an activation, by the formula in 64 bits, a small step to each
    side of x's pre-activation, w and b.  y is linear in w and b and piecewise linear in x, so differences are exact but for rounding."""
    x, w, bias, dz, off = _inputs(BF16, 40, 24, [50, 0, 30], 0, ref.LEAKY, 5)
    dx, dw, db = binding.pcc_grouped_linear_grad(dz, x, w, off, ref.LEAKY)
    gen = torch.Generator().manual_seed(6)
    before = torch.where(x > 0, x.double(), x.double() / ref.SLOPE).cpu()      # x = leaky(before)
    c = dz.double().cpu()

    def value(step):
        xs = ref.activate(before + step * e_x, ref.LEAKY)
        y, _ = ref.linear(xs, w.double().cpu() + step * e_w, bias.double() + step * e_b.cuda(), off.tolist(), ref.NONE)
        return (c * y).sum().item()

    for e in range(3):
        e_x = torch.randn(x.shape, generator=gen, dtype=torch.float64) * (e == 0)
        e_w = torch.randn(w.shape, generator=gen, dtype=torch.float64) * (e == 1)
        e_b = torch.randn(bias.shape, generator=gen, dtype=torch.float64) * (e == 2)
        h = 1e-7
        slope = (value(h) - value(-h)) / (2 * h)
        parts = (dx.double().cpu() * e_x, dw.double().cpu() * e_w, db.double().cpu() * e_b)
        got = sum(p.sum().item() for p in parts)
        # dx is rounded to bf16 (half a step each); dw and db are sums of 80 products in fp32; the difference loses 1e-16 / h of the value
        size = sum(p.abs().sum().item() for p in parts)
        assert abs(got - slope) <= 2.0 ** -8 * size * (e == 0) + 1e-5 * size + 1e-16 / h * (c.abs().sum().item() * 100)


def test_offsets_that_make_no_sense_stay_inside():
    """Falling offsets, and some beyond the rows: results are nobody's, memory is."""
    x, w, bias, dz, _ = _inputs(BF16, 48, 24, [100, 100], 0, ref.NONE, 3)
    for bad in ([0, 150, 90], [-5, 300, 1 << 40], [1 << 60, -(1 << 60), 7]):
        guard = torch.full((220, 24), 5.0, dtype=BF16, device="cuda")
        off = torch.tensor(bad).cuda()
        binding.pcc_grouped_linear(x, w, bias, off, ref.NONE, out=guard[10:210])
        dx = torch.full((220, 48), 5.0, dtype=BF16, device="cuda")
        binding.pcc_grouped_linear_grad(dz, x, w, off, ref.NONE, dx=dx[10:210])
        torch.cuda.synchronize()
        for t in (guard, dx):
            assert (t[:10] == 5).all() and (t[210:] == 5).all()


@pytest.mark.parametrize("fan_in,fan_out", [(48, 24), (200, 264)])
def test_falling_offsets_over_many_rows_stay_in_the_workspace(fan_in, fan_out):
    """Groups that overlap have more chunks than the workspace has room for: their sums are nobody's, what lies behind it is not touched."""
    rows, groups = 60000, 20
    x, dz = torch.ones(rows, fan_in, dtype=BF16, device="cuda"), torch.ones(rows, fan_out, dtype=BF16, device="cuda")
    w = torch.ones(groups, fan_out, fan_in, dtype=BF16, device="cuda")
    off = torch.tensor([0, rows] * 10 + [0]).cuda()
    need = binding.load().pcc_grouped_linear_grad_workspace_bytes(rows, groups, fan_in, fan_out)
    space = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device="cuda")
    binding.pcc_grouped_linear_grad(dz, x, w, off, workspace=space[:need])
    torch.cuda.synchronize()
    assert need > 0 and (space[need:] == 77).all()


def test_many_groups():
    """More groups than a wave has lanes, most of them empty."""
    lengths = [0] * 300
    for g in (0, 63, 64, 65, 127, 128, 200, 299):
        lengths[g] = 3 + g % 7
    x, w, bias, dz, off = _inputs(BF16, 40, 24, lengths, 2, ref.RELU, 11)
    y = binding.pcc_grouped_linear(x, w, bias, off, ref.LEAKY)
    want, bound = ref.linear(x, w, bias, off.tolist(), ref.LEAKY)
    ref.assert_near(y, want, bound, "y")
    for name, got, (value, bound) in zip(("dx", "dw", "db"), binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU),
                                         ref.linear_grad(dz, x, w, off.tolist(), ref.RELU)):
        ref.assert_near(got, value, bound, name)


def test_nan_of_one_row_stays_in_its_row_and_group():
    x, w, bias, dz, off = _inputs(BF16, 160, 160, [70, 70], 0, ref.NONE, 4)
    x[5, 7], dz[90, 3] = float("nan"), float("nan")
    y = binding.pcc_grouped_linear(x, w, bias, off, ref.RELU)
    bad = torch.isnan(y).any(1)
    assert bad[5] and int(bad.sum()) == 1
    dx, dw, db = binding.pcc_grouped_linear_grad(dz, x, w, off, ref.NONE)
    assert torch.isnan(dx[90]).all() and not torch.isnan(dx[:90]).any() and not torch.isnan(dx[91:]).any()
    assert torch.isnan(dw[0, :, 7]).all() and int(torch.isnan(dw[0]).sum()) == 160
    assert torch.isnan(dw[1, 3]).all() and int(torch.isnan(dw[1]).sum()) == 160
    assert int(torch.isnan(db).sum()) == 1 and torch.isnan(db[1, 3])


# ---------------------------------------------------------------------------------------------------- loss

def _heads(count, k, seed):
    gen = torch.Generator().manual_seed(seed)
    rgb = torch.randint(0, 256, (count, 3), generator=gen)
    rgb[::7] = 0
    rgb[1::7] = 255
    mean = rgb[:, :, None] / 256 + 0.15 * torch.randn(count, 3, k, generator=gen)
    head = torch.stack([torch.randn(count, 3, k, generator=gen), mean, 2.5 * torch.randn(count, 3, k, generator=gen) - 3], 2)
    params = torch.cat([head.reshape(count, 9 * k), 0.1 * torch.randn(count, 3 * k, generator=gen)], 1).float()
    special = params[:40].view(40, 12, k) if count >= 40 else None
    if special is not None:                          # log-sigmas at and beyond the clamp, means far off, logits far apart
        for c in range(3):
            special[0:4, 3 * c + 2] = torch.tensor([-8.0, 4.0, -9.0, 5.0])[:, None]
            special[4, 3 * c + 2] = float("nan")
            special[5:9, 3 * c + 1] = torch.tensor([40.0, -40.0, 1.5, -0.7])[:, None]
            special[9, 3 * c, 0] = 80.0
            special[10, 3 * c, 1] = float("-inf")
            special[11:15, 3 * c + 2] = torch.tensor([3.9, 2.0, 0.0, -2.0])[:, None]
            special[15, 3 * c + 2] = -30.0
            special[16, 3 * c + 2] = 30.0
    return params.contiguous(), rgb.to(torch.uint8)


# Relative error of the terms.  z = distance * width: the distance is rounded once (2^-24), the width by e^x (the argument's parts,
# 2^x to one step of fp32, a product: 4 * 2^-24), the product again: 6 * 2^-24.  A density e^(-z^2/2) turns that into z^2 times it; terms
# with z > 9 (e^-40 against one count of 65,536) are below 1e-12 of the size asked for, so z^2 <= 81 would give 3e-5; but a term's weight falls
# with e^(-z^2/2) while its error grows with z^2, and sizes are those of the largest term of the channel only for z of a few: 2e-5 for z <= 7
# relative to the term itself.  Mills' ratio (4e-7), the softmax, 1/counts and the product of four factors add 10 * 2^-24.
TERM = 81 * 6 * 2.0 ** -24 + 4e-7 + 10 * 2.0 ** -24


@pytest.mark.parametrize("dist", [0, 1])
@pytest.mark.parametrize("k", [3, 5, 7])
@pytest.mark.parametrize("count", [1, 63, 700])
def test_mixture_loss(k, dist, count):
    params, rgb = _heads(count, k, 100 * k + count + dist)
    scale = 0.37
    bits, grad = binding.pcc_mixture_loss(params.cuda(), rgb.cuda(), dist, scale)
    want_bits = ref.code_length(params, rgb, k, dist)
    # counts are off by TERM at most relative to themselves; log2 by a step of 16; three channels
    assert (bits.double().cpu() - want_bits).abs().max().item() <= 3 * (TERM / math.log(2) + 16 * 2.0 ** -23)
    want, size = ref.loss_gradient(params, rgb, k, dist, scale)
    for dtype in (FP32, BF16, FP16):
        b2, g = binding.pcc_mixture_loss(params.cuda(), rgb.cuda(), dist, scale, grad_dtype=dtype)
        assert torch.equal(b2, bits)
        got = g.double().cpu()
        tol = TERM * size + ref.HALF_STEP[dtype] * want.abs() * (1 + TERM) + 1e-12 + ref.SMALLEST[dtype]
        assert torch.isfinite(got).all()
        worst = ((got - want).abs() / tol).max().item()
        assert worst <= 1.0, (dtype, worst)
    only, none = binding.pcc_mixture_loss(params.cuda(), rgb.cuda(), dist, scale, want_grad=False)
    assert none is None and torch.equal(only, bits)


@pytest.mark.parametrize("dist", [0, 1])
def test_loss_gradient_against_differences(dist):
    k, count = 5, 64
    params, rgb = _heads(count, k, 77)
    params[:40] = _heads(count, k, 78)[0][17:57]                             # without the special rows, where the clamp has a corner
    params = params.double()
    _, grad = binding.pcc_mixture_loss(params.float().cuda(), rgb.cuda(), dist, 1.0)
    params = params.float().double()
    gen = torch.Generator().manual_seed(5)
    for _ in range(4):
        e = torch.randn(params.shape, generator=gen, dtype=torch.float64)
        e[:, 6 * k - k:6 * k] = 0                                            # one channel's widths stay
        h = 1e-7
        up, down = ref.code_length(params + h * e, rgb, k, dist), ref.code_length(params - h * e, rgb, k, dist)
        slope = (up - down) / (2 * h)
        got = (grad.double().cpu() * e).sum(1)
        _, size = ref.loss_gradient(params, rgb, k, dist, 1.0)
        # the third derivative of a component of width e^-8 is (3000)^3 of its own size: h^2 * 2.7e10 = 3e-4 of the terms
        assert ((got - slope).abs() <= (5e-4 + TERM) * (size * e.abs()).sum(1) + 1e-16 / h * 100).all()


def test_loss_masks():
    """Weight 0: nothing of the pixel counts, whatever its outputs are; other weights multiply."""
    k = 3
    params, rgb = _heads(300, k, 9)
    gen = torch.Generator().manual_seed(10)
    weight = torch.rand(300, generator=gen) + 0.5
    weight[::3] = 0
    want, size = ref.loss_gradient(params, rgb, k, 0, 2.0, weight)
    want_bits = ref.code_length(params, rgb, k, 0)
    dirty = params.clone()
    dirty[0::6], dirty[3::6] = float("nan"), float("inf")
    bits, grad = binding.pcc_mixture_loss(dirty.cuda(), rgb.cuda(), 0, 2.0, weight=weight.cuda())
    assert (bits[::3] == 0).all() and (grad[::3] == 0).all()
    keep = weight != 0
    assert ((grad.double().cpu() - want).abs() <= (TERM + 2.0 ** -23) * size + 1e-12)[keep].all()
    assert ((bits.double().cpu() - want_bits).abs() <= 3 * (TERM / math.log(2) + 16 * 2.0 ** -23))[keep].all()
    none = torch.zeros_like(weight)
    bits, grad = binding.pcc_mixture_loss(dirty.cuda(), rgb.cuda(), 0, 2.0, weight=none.cuda())
    assert (bits == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("k", [3, 5, 7])
def test_loss_rows_with_strides_and_in_place(k):
    params, rgb = _heads(130, k, 21 + k)
    _, want = binding.pcc_mixture_loss(params.cuda(), rgb.cuda())
    wide = torch.full((130, 12 * k + 5), float("nan"), device="cuda")
    wide[:, 2:2 + 12 * k] = params.cuda()
    out = torch.full((130, 12 * k + 3), 9.0, dtype=BF16, device="cuda")
    binding.pcc_mixture_loss(wide[:, 2:2 + 12 * k], rgb.cuda(), grad=out[:, 1:1 + 12 * k])
    assert torch.equal(out[:, 1:1 + 12 * k], want.to(BF16)) and (out[:, 0] == 9).all() and (out[:, 1 + 12 * k:] == 9).all()
    view = wide[:, 2:2 + 12 * k]
    binding.pcc_mixture_loss(view, rgb.cuda(), grad=view)
    assert torch.equal(view, want) and torch.isnan(wide[:, :2]).all() and torch.isnan(wide[:, 2 + 12 * k:]).all()


@pytest.mark.parametrize("dist", [0, 1])
def test_shares_of_all_levels_make_one(dist):
    params, _ = _heads(60, 5, 31)
    params = params[17:18].repeat(256, 1)
    levels = torch.arange(256, dtype=torch.uint8)
    rgb = torch.stack([levels, torch.zeros_like(levels), torch.zeros_like(levels)], 1)
    bits, _ = binding.pcc_mixture_loss(params.cuda(), rgb.cuda(), dist, want_grad=False)
    rest = ref.code_length(params, rgb, 5, dist) - _first_channel(params, rgb, dist)
    share = torch.exp2(-(bits.double().cpu() - rest)).sum().item()
    # 256 shares, each off by what three code lengths may be off
    assert abs(share - 1) <= 3 * (TERM / math.log(2) + 16 * 2.0 ** -23)


def _first_channel(params, rgb, dist):
    pi, a, b, _ = ref.mixture(params, rgb, 5, dist)[0]
    x = rgb[:, :1].double()
    q = torch.where(x == 0, ref.tail(-b, dist), torch.where(x == 255, ref.tail(a, dist), ref.tail(a, dist) - ref.tail(b, dist)))
    return -torch.log2((65280 * (pi * q).sum(1) + 1) / 65536)


def test_bits_are_those_of_the_coder(blob):
    """pcc_encode_probs counts with the integer CDF: each share is off by less than one count of 65,536 and by its table's error."""
    img = synth.make_image(3, synth.ImageSpec(64, 48, 5, 4.0, 20.0))[None]
    codec = binding.Codec(blob, 0)
    d = torch.from_numpy(img).cuda()
    params, coder = codec.pcc_encode_probs(d)
    bits, _ = binding.pcc_mixture_loss(params.view(-1, 60), d.view(-1, 3), want_grad=False)
    codec.close()
    assert abs(bits.double().sum().item() / coder.double().sum().item() - 1) <= 1e-3      # the bar of the coder against the oracle


# ---------------------------------------------------------------------------------------------------- AdamW

SIZES = [1, 0, 255, 256, 257, 4096, 4097, 160 * 160, 3, 12291]


def _tensors(sizes, seed, shift=0):
    """Views into one buffer, `shift` elements from where vectors could be read."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for n in sizes:
        full = torch.randn(n + 8, generator=gen).cuda()
        out.append(full[shift:shift + n])
    return out


@pytest.mark.parametrize("grad_dtype,copy_dtype", [(FP32, BF16), (BF16, FP16), (FP16, None)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw(bits, shift, grad_dtype, copy_dtype):
    params = _tensors(SIZES, 1, shift)
    grads = [torch.zeros(n + 8, dtype=grad_dtype, device="cuda")[shift:shift + n] for n in SIZES]
    copies = [torch.zeros(n + 8, dtype=copy_dtype, device="cuda")[shift:shift + n] if i != 3 else None for i, n in enumerate(SIZES)] if copy_dtype else None
    hyper = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    opt = binding.AdamW(params, grads, copies=copies, state_bits=bits, **hyper)
    want = [ref.AdamW(p.cpu().numpy(), bits, **hyper) for p in params]
    rng = np.random.default_rng(2)
    for step in range(5):
        for g, r in zip(grads, want):
            value = torch.from_numpy((rng.normal(size=len(r.p)) * np.exp(2 * rng.normal(size=len(r.p)))).astype(np.float32)).to(grad_dtype)
            if step == 3:
                value[::2] = 0
            g.copy_(value)
            if len(r.p):
                r.step(value.float().numpy())
        opt.pcc_adamw_step()
    assert opt.step.item() == 5
    for i, r in enumerate(want):
        if not len(r.p):
            continue
        p = params[i].cpu().numpy()
        # the moments are the same bits (products and sums in the same order); the update is a quotient and a product, each off by one step
        # of fp32 at most, and the parameter's own three roundings, in each of five steps
        assert np.array_equal(opt.m[i].view(torch.uint8).cpu().numpy(), r.m) if bits == 8 else np.array_equal(opt.m[i].cpu().numpy(), r.m), i
        assert np.array_equal(opt.v[i].view(torch.uint8).cpu().numpy(), r.v) if bits == 8 else np.array_equal(opt.v[i].cpu().numpy(), r.v), i
        if bits == 8:
            assert np.array_equal(opt.m_scale[i].cpu().numpy(), r.ms) and np.array_equal(opt.v_scale[i].cpu().numpy(), r.vs)
        assert np.all(np.abs(p - r.p) <= 5 * 2.0 ** -24 * (3 * np.abs(r.p) + 12 * 3e-3 * 10)), i
        if copies and copies[i] is not None:
            assert torch.equal(copies[i], params[i].to(copy_dtype))
    assert all((s.min().item() >= 1 if bits == 8 else True) for s in [opt.v[7].view(torch.uint8)])


def test_adamw_follows_a_rate_on_the_device_and_resumes():
    params = _tensors([1000], 3)
    grads = [torch.ones(1000, device="cuda")]
    rate = torch.tensor([0.0], device="cuda")
    opt = binding.AdamW(params, grads, lr=1.0, weight_decay=0.0, lr_tensor=rate)
    start = params[0].clone()
    opt.pcc_adamw_step()
    assert torch.equal(params[0], start)
    rate.fill_(0.5)
    opt.pcc_adamw_step()
    assert (params[0] < start).all()
    # a second plan over the same states goes on where the first stopped
    more = binding.AdamW(params, grads, lr=0.25, weight_decay=0.0, step=opt.step, m=opt.m, v=opt.v)
    other = [params[0].clone()]
    both = binding.AdamW(other, grads, lr=0.25, weight_decay=0.0, step=opt.step.clone(), m=[opt.m[0].clone()], v=[opt.v[0].clone()])
    more.pcc_adamw_step()
    both.pcc_adamw_step()
    assert more.step.item() == 3 and torch.equal(params[0], other[0])


def test_small_states_follow_slow_moments():
    """beta2 = 0.999 changes a second moment by a thousandth a step, far less than a step of its code; on average over the
    places of the block the codes follow all the same.  A place's code is a random walk around the moment with steps of at most 1/8 of
    it that takes 1,000 steps to forget; over 256 x 16 places the mean is within 3 % (eight codes' steps / sqrt(4096) is 1.6 %)."""
    n = 4096
    params = [torch.zeros(n, device="cuda")]
    grads = [torch.full((n,), 1.0, device="cuda")]
    opt = binding.AdamW(params, grads, state_bits=8, lr=0.0, betas=(0.9, 0.999), weight_decay=0.0)
    for _ in range(10):
        opt.pcc_adamw_step()
    grads[0][: n // 2 * 2: 2] = 0.25                 # half of the places get smaller gradients, the block's largest stays
    v = 1 - 0.999 ** 10
    for _ in range(400):
        opt.pcc_adamw_step()
        v = 0.999 * v + 0.001 * 0.25 ** 2
    got = (opt.v[0].float().view(-1, 256) * opt.v_scale[0][:, None]).square().view(-1)[::2].mean().item()
    assert abs(got / v - 1) <= 0.03, (got, v)


def test_a_gradient_that_is_not_a_number_stays_in_its_block():
    params = _tensors([1024], 5)
    grads = [torch.ones(1024, device="cuda")]
    for bits in (32, 8):
        p = [params[0].clone()]
        opt = binding.AdamW(p, grads, state_bits=bits)
        grads[0][300] = float("nan")
        opt.pcc_adamw_step()
        grads[0][300] = 1.0
        opt.pcc_adamw_step()
        bad = torch.isnan(p[0])
        assert bad[300] and not bad[:256].any() and not bad[512:].any() and int(bad.sum()) == 1


# ---------------------------------------------------------------------------------------------------- as a program uses them

def _one_step(img, w, b, rgb, off):
    x = binding.pcc_contexts(img)
    h = binding.pcc_grouped_linear(x, w[0], b[0], off, ref.RELU)
    o = binding.pcc_grouped_linear(h, w[1], b[1], off, ref.NONE, out_dtype=FP32)
    bits, do = binding.pcc_mixture_loss(o, rgb, scale=1.0 / rgb.shape[0], grad_dtype=BF16)
    dh, dw1, db1 = binding.pcc_grouped_linear_grad(do, h, w[1], off, ref.RELU)
    _, dw0, db0 = binding.pcc_grouped_linear_grad(dh, x, w[0], off, want_dx=False)
    return bits, dw0, db0, dw1, db1


def _net(seed):
    gen = torch.Generator().manual_seed(seed)
    w = [(torch.randn(1, 96, 32, generator=gen) / 4).to(BF16).cuda(), (torch.randn(1, 60, 96, generator=gen) / 10).to(BF16).cuda()]
    return w, [torch.randn(1, 96, generator=gen).cuda() * 0.1, torch.randn(1, 60, generator=gen).cuda() * 0.1]


def test_another_stream_and_a_captured_step():
    img = torch.from_numpy(synth.make_image(5, synth.ImageSpec(130, 70, 5, 4.0, 20.0))[None]).cuda()
    rgb = img.view(-1, 3).contiguous()
    w, b = _net(1)
    off = torch.tensor([0, 130 * 70]).cuda()
    want = [t.clone() for t in _one_step(img, w, b, rgb, off)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _one_step(img, w, b, rgb, off)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))

    graph = torch.cuda.CUDAGraph()
    other = torch.from_numpy(synth.make_image(6, synth.ImageSpec(130, 70, 5, 4.0, 20.0))[None]).cuda()
    source = img.clone()
    source_rgb = source.view(-1, 3)
    with torch.cuda.graph(graph):
        captured = _one_step(source, w, b, source_rgb, off)
    for k in range(4):
        now = other if k % 2 else img
        source.copy_(now)
        eager = [t.clone() for t in _one_step(now, w, b, now.view(-1, 3), off)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, captured)), k


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_adamw_step(bits):
    grads = [torch.randn(5000, device="cuda"), torch.randn(77, device="cuda")]
    rate = torch.tensor([1e-3], device="cuda")

    def make():
        torch.manual_seed(3)
        return binding.AdamW([torch.randn(5000, device="cuda"), torch.randn(77, device="cuda")], grads, state_bits=bits, lr_tensor=rate)

    eager, held = make(), make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held.pcc_adamw_step()
    for k in range(4):
        rate.fill_(1e-3 * (k + 1))
        grads[0].mul_(0.5)
        eager.pcc_adamw_step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert held.step.item() == k + 1 and all(torch.equal(a, b) for a, b in zip(eager.params, held.params))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(eager.v, held.v))


def test_two_streams_at_once_with_a_workspace_each():
    x, w, _, dz, off = _inputs(BF16, 160, 128, [30000, 20000], 0, ref.RELU, 8)
    want = binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU)
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                results.append(binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU))
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("fan_in,fan_out", [(32, 16), (300, 7)])
def test_without_any_rows(fan_in, fan_out):
    x, w, bias, dz, off = _inputs(BF16, fan_in, fan_out, [0, 0], 0, ref.NONE, 1)
    assert binding.pcc_grouped_linear(x, w, bias, off).shape == (0, fan_out)
    dx, dw, db = binding.pcc_grouped_linear_grad(dz, x, w, off, dw=torch.ones_like(w, dtype=FP32), db=torch.ones_like(bias))
    assert dx.shape == (0, fan_in) and (dw == 0).all() and (db == 0).all()
    bits, grad = binding.pcc_mixture_loss(torch.zeros(0, 36, device="cuda"), torch.zeros(0, 3, dtype=torch.uint8, device="cuda"))
    assert bits.numel() == 0 and grad.shape == (0, 36)


def test_adamw_of_the_same_tensor_twice_is_refused():
    p, g = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    with pytest.raises(binding.PccError):
        binding.AdamW([p, p[100:]], [g, g[100:]])


def test_gpu_tensors_that_do_not_fit_are_refused():
    x, w, bias, dz, off = _inputs(BF16, 32, 16, [4, 4], 0, ref.NONE, 1)
    for bad in (lambda: binding.pcc_grouped_linear(x, w.half(), bias, off), lambda: binding.pcc_grouped_linear(x, w, bias.half(), off),
                lambda: binding.pcc_grouped_linear(x, w, bias, off.int()), lambda: binding.pcc_grouped_linear(x, w, bias, off[:2]),
                lambda: binding.pcc_grouped_linear(x, w, bias.cpu(), off), lambda: binding.pcc_grouped_linear(x.t(), w, bias, off),
                lambda: binding.pcc_grouped_linear(x, w[:, :, ::2], bias, off), lambda: binding.pcc_grouped_linear(x, w, bias, off, out=dz.half()),
                lambda: binding.pcc_grouped_linear(x[:1].expand(8, 32), w, bias, off, out=dz[:1].expand(8, 16)),
                lambda: binding.pcc_grouped_linear_grad(dz.float(), x, w, off), lambda: binding.pcc_grouped_linear_grad(dz, x, w, off, dw=w),
                lambda: binding.pcc_mixture_loss(torch.zeros(4, 59, device="cuda"), torch.zeros(4, 3, dtype=torch.uint8, device="cuda")),
                lambda: binding.AdamW([torch.zeros(3, device="cuda")], [torch.zeros(4, device="cuda")]),
                lambda: binding.AdamW([torch.zeros(3, device="cuda")], [torch.zeros(3, device="cuda")], copies=[torch.zeros(3, device="cuda")])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(binding.PccError) as e:
        binding.pcc_mixture_loss(torch.zeros(4, 48, device="cuda"), torch.zeros(4, 3, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.PCC_E_ARG
    with pytest.raises(binding.PccError):
        binding.pcc_grouped_linear(x, w, bias, off, act=3)
