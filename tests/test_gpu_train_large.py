"""Paths of the training operators that only large calls take.  Needs an MI355X."""
import math

import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2212_01185_amd import binding

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


# ---------------------------------------------------------------------------------------------------- products in tiles of 256

def _view(t, before, behind):
    """t on the GPU as columns of a wider buffer of NaN."""
    full = torch.full((t.shape[0], before + t.shape[1] + behind), float("nan"), dtype=t.dtype)
    full[:, before:before + t.shape[1]] = t
    return full.cuda()[:, before:before + t.shape[1]]


# Rows of x begin at even elements (with whole chunks of eight, and with one cut by the row's end) or at odd ones; those of the result in
# whole pieces or not.  Groups of 9,000 and 8,000 rows with an empty one between, and rows of no group behind: 512 rows a group and
# 256 tiles at least are what the launch wants.
@pytest.mark.parametrize("fan_in,fan_out,dtype,out_dtype,x_pad,y_pad,act,with_bias", [
    (256, 1030, BF16, BF16, (0, 0), (0, 2), ref.RELU, True), (250, 1030, FP16, FP32, (0, 0), (0, 0), ref.LEAKY, True),
    (250, 1030, BF16, BF16, (2, 4), (4, 2), ref.NONE, False), (250, 1032, FP16, FP16, (0, 0), (1, 2), ref.RELU, True),
    (263, 1030, FP16, FP32, (0, 0), (0, 2), ref.NONE, True), (264, 1030, BF16, FP32, (1, 0), (0, 0), ref.LEAKY, True),
    (63, 1031, BF16, BF16, (0, 1), (0, 0), ref.RELU, False), (1000, 900, FP16, FP16, (0, 8), (0, 0), ref.RELU, True)])
def test_forward_in_large_tiles(fan_in, fan_out, dtype, out_dtype, x_pad, y_pad, act, with_bias):
    lengths, tail = [9000, 0, 8000], 3
    rows, groups = sum(lengths) + tail, len(lengths)
    assert rows // groups >= 512 and (rows // 256 + groups) * (-(-fan_out // 256)) >= 256
    gen = torch.Generator().manual_seed(fan_in + fan_out)
    x = torch.randn(rows, fan_in, generator=gen).to(dtype)
    x[-tail:] = float("nan")
    w = (torch.randn(groups, fan_out, fan_in, generator=gen) / math.sqrt(fan_in)).to(dtype)
    bias = torch.randn(groups, fan_out, generator=gen) if with_bias else None
    offsets = [0] + np.cumsum(lengths).tolist()
    full = torch.full((rows, y_pad[0] + fan_out + y_pad[1]), 5.0, dtype=out_dtype, device="cuda")
    out = full[:, y_pad[0]:y_pad[0] + fan_out]
    got = binding.pcc_grouped_linear(_view(x, *x_pad), w.cuda(), bias.cuda() if with_bias else None, torch.tensor(offsets).cuda(), act, out=out)
    want, bound = ref.linear(x, w, bias, offsets, act)
    ref.assert_near(got, want, bound, (fan_in, fan_out))
    assert (got[-tail:] == 5).all() and (full[:, :y_pad[0]] == 5).all() and (full[:, y_pad[0] + fan_out:] == 5).all()


# ---------------------------------------------------------------------------------------------------- sums of many groups

@pytest.mark.parametrize("fan_in,fan_out", [(48, 24), (200, 264)])
def test_sums_of_cut_groups_behind_many_others(fan_in, fan_out):
    """Groups of several chunks before and behind the 64th and 128th: their sums are numbered over all groups in front."""
    lengths = [7 * (g % 5) for g in range(150)]
    for g in (0, 3, 63, 64, 70, 127, 128, 149):
        lengths[g] = 4000 + 100 * (g % 7)
    gen = torch.Generator().manual_seed(9)
    rows = sum(lengths)
    x, dz = torch.randn(rows, fan_in, generator=gen).to(BF16), torch.randn(rows, fan_out, generator=gen).to(BF16)
    w = (torch.randn(150, fan_out, fan_in, generator=gen) / math.sqrt(fan_in)).to(BF16)
    offsets = [0] + np.cumsum(lengths).tolist()
    first = binding.pcc_grouped_linear_grad(dz.cuda(), x.cuda(), w.cuda(), torch.tensor(offsets).cuda(), ref.RELU)
    for name, got, (value, bound) in zip(("dx", "dw", "db"), first, ref.linear_grad(dz, x, w, offsets, ref.RELU)):
        ref.assert_near(got, value, bound, name)
    again = binding.pcc_grouped_linear_grad(dz.cuda(), x.cuda(), w.cuda(), torch.tensor(offsets).cuda(), ref.RELU)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


# ---------------------------------------------------------------------------------------------------- AdamW

SIZES = [9_000_001, 4097, 8_000_003, 255, 300_000]     # 17.3 million: pieces of four blocks a wave, and more of them than workgroups
APART = 1 << 21                                         # elements of a plan that has pieces of one block a wave


@pytest.mark.parametrize("grad_dtype", [FP32, BF16])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_many_elements(bits, shift, grad_dtype):
    """Every element has the bits that it has in a plan of few elements; some stretches are compared with the reference as well."""
    gen = torch.Generator(device="cuda").manual_seed(bits + shift)
    hyper = dict(lr=1e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    make = lambda n, dtype: torch.randn(n + 8, generator=gen, device="cuda").to(dtype)[shift:shift + n]  # noqa: E731
    params, grads = [make(n, FP32) for n in SIZES], [make(n, grad_dtype) for n in SIZES]
    copies = [torch.zeros(n + 8, dtype=BF16, device="cuda")[shift:shift + n] for n in SIZES]
    start = [p.clone() for p in params]
    opt = binding.AdamW(params, grads, copies=copies, state_bits=bits, **hyper)
    spans = [(i, a, min(a + APART, n)) for i, n in enumerate(SIZES) for a in range(0, n, APART)]
    few_grads = [torch.empty(b - a, dtype=grad_dtype, device="cuda") for _, a, b in spans]
    few = [binding.AdamW([start[i][a:b].clone()], [g], copies=[torch.zeros(b - a, dtype=BF16, device="cuda")], state_bits=bits, **hyper)
           for (i, a, b), g in zip(spans, few_grads)]
    # stretches of two blocks: at the ends of tensors, at a piece's end, where a workgroup takes its second piece
    looked_at = [(i, a) for i, n in enumerate(SIZES) for a in (0, 4096 - 256, 1024 * 4096 - 256, 4096 * 1024 + 4096 - 256, n // 256 * 256 - 256) if 0 <= a < n]
    want = [ref.AdamW(start[i][a:a + 512].cpu().numpy(), bits, **hyper) for i, a in looked_at]
    for _ in range(3):
        for g in grads:
            g.copy_(torch.randn(g.shape, generator=gen, device="cuda"))
        for (i, a, b), g, one in zip(spans, few_grads, few):
            g.copy_(grads[i][a:b])
            one.pcc_adamw_step()
        opt.pcc_adamw_step()
        for (i, a), r in zip(looked_at, want):
            r.step(grads[i][a:a + 512].float().cpu().numpy())
    for (i, a, b), one in zip(spans, few):
        pairs = [(params[i], one.params[0]), (copies[i], one.copies[0]), (opt.m[i], one.m[0]), (opt.v[i], one.v[0])]
        assert all(torch.equal(x[a:b].view(torch.uint8) if x.element_size() == 1 else x[a:b], y.view(torch.uint8) if y.element_size() == 1 else y)
                   for x, y in pairs), (i, a)
        if bits == 8:
            blocks = slice(a // 256, -(-b // 256))
            assert torch.equal(opt.m_scale[i][blocks], one.m_scale[0]) and torch.equal(opt.v_scale[i][blocks], one.v_scale[0]), (i, a)
    for (i, a), r in zip(looked_at, want):
        m, v = (t[i][a:a + 512] for t in (opt.m, opt.v))
        assert np.array_equal((m.view(torch.uint8) if bits == 8 else m).cpu().numpy(), r.m), (i, a)
        assert np.array_equal((v.view(torch.uint8) if bits == 8 else v).cpu().numpy(), r.v), (i, a)
        # in each of three steps the quotient and the product, each off by a step of fp32 at most on an update of ten rates at most, and the
        # parameter's own three roundings
        assert np.all(np.abs(params[i][a:a + 512].cpu().numpy() - r.p) <= 3 * 2.0 ** -24 * (3 * np.abs(r.p) + 12 * hyper["lr"] * 10)), (i, a)


def test_adamw_behind_the_four_billionth_element():
    n, tail = (1 << 32) + 70000, 70000 + 4096
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    p[-tail:] = torch.randn(tail, generator=gen, device="cuda")
    g[-tail:] = torch.randn(tail, generator=gen, device="cuda").to(BF16)
    few = [p[-tail:].clone()]
    opt, one = binding.AdamW([p], [g], state_bits=8), binding.AdamW(few, [g[-tail:].clone()], state_bits=8)
    for _ in range(2):
        opt.pcc_adamw_step()
        one.pcc_adamw_step()
    assert torch.equal(p[-tail:], few[0]) and not p[:1 << 20].any()
    for a, b in ((opt.m[0], one.m[0]), (opt.v[0], one.v[0])):
        assert torch.equal(a[-tail:].view(torch.uint8), b.view(torch.uint8))


# ---------------------------------------------------------------------------------------------------- rows far apart

def _apart(t, ld=1 << 15):
    """t's values in rows `ld` elements apart: the last ones lie behind the 2^32nd element."""
    full = torch.empty((t.shape[0], ld), dtype=t.dtype, device="cuda")
    assert t.shape[0] * ld > 1 << 32
    full[:, :t.shape[1]] = t
    return full[:, :t.shape[1]]


@pytest.mark.parametrize("fan_in,fan_out", [(32, 48), (200, 264), (201, 264)])
def test_products_of_rows_far_apart(fan_in, fan_out):
    rows = (1 << 17) + 600
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dz = (torch.randn(rows, n, generator=gen, device="cuda").to(BF16) for n in (fan_in, fan_out))
    w, off = torch.randn(2, fan_out, fan_in, generator=gen, device="cuda").to(BF16), torch.tensor([0, 100, rows], device="cuda")
    ld = 1 << 15
    y = torch.empty((rows, ld), dtype=FP32, device="cuda")[:, :fan_out]
    got = binding.pcc_grouped_linear(_apart(x), w, None, off, ref.RELU, out=y)
    assert torch.equal(got, binding.pcc_grouped_linear(x.contiguous(), w, None, off, ref.RELU, out_dtype=FP32))
    del y, got
    dx = torch.empty((rows, ld), dtype=BF16, device="cuda")[:, :fan_in]
    far, near = binding.pcc_grouped_linear_grad(_apart(dz), _apart(x), w, off, ref.RELU, dx=dx), binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU)
    if fan_in % 2 == 0:                 # odd rows one behind the other take other loads, and the same order of sums
        assert all(torch.equal(a, b) for a, b in zip(far, near))
    want = ref.linear_grad(dz[-500:], x[-500:], w[1:], [0, 500], ref.RELU)[0]
    ref.assert_near(far[0][-500:], *want, "dx")


def test_contexts_and_loss_of_rows_far_apart():
    img = torch.randint(0, 256, (1, 260, 600, 3), dtype=torch.uint8, device="cuda")
    rows = 260 * 600
    far = torch.empty((rows, 1 << 15), dtype=BF16, device="cuda")[:, :40]
    assert torch.equal(binding.pcc_contexts(img, 12, 3, 40, out=far), binding.pcc_contexts(img, 12, 3, 40))
    del far
    params = torch.randn(rows, 60, device="cuda")
    near = binding.pcc_mixture_loss(params, img.view(-1, 3), grad_dtype=FP16)
    grad = torch.empty((rows, 1 << 15), dtype=FP16, device="cuda")[:, :60]
    far = binding.pcc_mixture_loss(_apart(params), img.view(-1, 3), grad=grad)
    assert torch.equal(near[0], far[0]) and torch.equal(near[1], far[1])


# ---------------------------------------------------------------------------------------------------- all the groups there may be

def test_as_many_groups_as_there_may_be():
    groups, fan_in, fan_out = 65535, 8, 6
    gen = torch.Generator().manual_seed(5)
    lengths = torch.randint(0, 3, (groups,), generator=gen)
    lengths[40000] = 3000
    lengths[-1] = 1
    offsets = torch.nn.functional.pad(lengths.cumsum(0), (1, 0))
    rows = int(offsets[-1])
    x, dz = torch.randn(rows, fan_in, generator=gen).to(BF16), torch.randn(rows, fan_out, generator=gen).to(BF16)
    w = torch.randn(groups, fan_out, fan_in, generator=gen).to(BF16)
    bias = torch.randn(groups, fan_out, generator=gen)
    of = torch.repeat_interleave(torch.arange(groups), lengths)
    y = binding.pcc_grouped_linear(x.cuda(), w.cuda(), bias.cuda(), offsets.cuda(), out_dtype=FP32)
    want, size = torch.zeros(rows, fan_out, dtype=torch.float64), torch.zeros(rows, fan_out, dtype=torch.float64)
    for k in range(fan_in):
        want += x[:, k:k + 1].double() * w[of, :, k].double()
        size += (x[:, k:k + 1].double() * w[of, :, k].double()).abs()
    ref.assert_near(y, want + bias[of].double(), (fan_in + 3) * ref.EPS32 * (size + bias[of].abs().double()), "y")
    dx, dw, db = binding.pcc_grouped_linear_grad(dz.cuda(), x.cuda(), w.cuda(), offsets.cuda())
    want, size = torch.zeros(rows, fan_in, dtype=torch.float64), torch.zeros(rows, fan_in, dtype=torch.float64)
    for k in range(fan_out):
        want += dz[:, k:k + 1].double() * w[of, k].double()
        size += (dz[:, k:k + 1].double() * w[of, k].double()).abs()
    ref.assert_near(dx, want, (fan_out + 2) * ref.EPS32 * size, "dx")
    terms = dz[:, :, None].double() * x[:, None].double()
    sums, sizes = torch.zeros(w.shape, dtype=torch.float64).index_add_(0, of, terms), torch.zeros(w.shape, dtype=torch.float64).index_add_(0, of, terms.abs())
    ref.assert_near(dw, sums, (lengths + 2).double()[:, None, None] * ref.EPS32 * sizes, "dw")
    sums = torch.zeros(groups, fan_out, dtype=torch.float64).index_add_(0, of, dz.double())
    sizes = torch.zeros(groups, fan_out, dtype=torch.float64).index_add_(0, of, dz.double().abs())
    ref.assert_near(db, sums, (lengths + 2).double()[:, None] * ref.EPS32 * sizes, "db")


@pytest.mark.parametrize("fan_in,fan_out", [(32, 32), (200, 8)])
def test_time_does_not_grow_with_the_square_of_groups(fan_in, fan_out):
    """As many groups as there may be, of a row each: 130 ms when every workgroup read all offsets, under 1 ms since."""
    groups = 65535
    x, w = torch.ones(groups, fan_in, dtype=BF16, device="cuda"), torch.ones(groups, fan_out, fan_in, dtype=BF16, device="cuda")
    off = torch.arange(groups + 1, device="cuda")
    dz = torch.ones(groups, fan_out, dtype=BF16, device="cuda")
    for call in (lambda: binding.pcc_grouped_linear(x, w, None, off), lambda: binding.pcc_grouped_linear_grad(dz, x, w, off)):
        times = []
        for _ in range(4):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            call()
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end))
        assert min(times) < 20


@pytest.mark.parametrize("fan_in,fan_out", [(48, 24), (200, 264)])
@pytest.mark.parametrize("kind", ["overlap", "fall", "beyond"])
def test_offsets_of_many_groups_that_make_no_sense_stay_inside(fan_in, fan_out, kind):
    rows, groups = 30000, 130
    off = {"overlap": torch.tensor([0, rows] * 65 + [0]), "fall": torch.linspace(rows, 0, groups + 1).long(),
           "beyond": torch.tensor([-5, 1 << 60, 7, -(1 << 60), 40] * 26 + [1 << 40])}[kind].cuda()
    x, dz = torch.ones(rows, fan_in, dtype=BF16, device="cuda"), torch.ones(rows, fan_out, dtype=BF16, device="cuda")
    w = torch.ones(groups, fan_out, fan_in, dtype=BF16, device="cuda")
    y, dx = (torch.full((rows + 20, n), 5.0, dtype=BF16, device="cuda") for n in (fan_out, fan_in))
    need = binding.load().pcc_grouped_linear_grad_workspace_bytes(rows, groups, fan_in, fan_out)
    space = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device="cuda")
    binding.pcc_grouped_linear(x, w, None, off, out=y[10:-10])
    binding.pcc_grouped_linear_grad(dz, x, w, off, dx=dx[10:-10], workspace=space[:need])
    torch.cuda.synchronize()
    assert need > 0 and (space[need:] == 77).all() and all((t[:10] == 5).all() and (t[-10:] == 5).all() for t in (y, dx))


@pytest.mark.parametrize("fan_in,fan_out", [(48, 24), (200, 264)])
@pytest.mark.parametrize("first", [0, 1, 5000])
def test_more_than_64_groups_behind_rows_of_none(fan_in, fan_out, first):
    """The first group need not begin at the first row; more than 64 groups are found by their offsets."""
    lengths = [(37 * g) % 90 for g in range(200)]
    lengths[11], lengths[120] = 1500, 2300
    offsets = (first + np.concatenate([[0], np.cumsum(lengths)])).tolist()
    rows = offsets[-1] + 700
    gen = torch.Generator().manual_seed(first)
    x, dz = torch.randn(rows, fan_in, generator=gen).to(BF16), torch.randn(rows, fan_out, generator=gen).to(BF16)
    w = (torch.randn(200, fan_out, fan_in, generator=gen) / math.sqrt(fan_in)).to(BF16)
    nobody = torch.ones(rows, dtype=torch.bool)
    nobody[offsets[0]:offsets[-1]] = False
    x[nobody], dz[nobody] = float("nan"), float("inf")
    y, dx = (torch.full((rows, n), 5.0, dtype=BF16, device="cuda") for n in (fan_out, fan_in))
    off = torch.tensor(offsets).cuda()
    binding.pcc_grouped_linear(x.cuda(), w.cuda(), None, off, ref.RELU, out=y)
    _, dw, db = binding.pcc_grouped_linear_grad(dz.cuda(), x.cuda(), w.cuda(), off, ref.LEAKY, dx=dx)
    ref.assert_near(y, *ref.linear(x, w, None, offsets, ref.RELU), "y")
    for name, got, (value, bound) in zip(("dx", "dw", "db"), (dx, dw, db), ref.linear_grad(dz, x, w, offsets, ref.LEAKY)):
        ref.assert_near(got, value, bound, name)
    assert (y[nobody.cuda()] == 5).all() and (dx[nobody.cuda()] == 5).all()


# ---------------------------------------------------------------------------------------------------- the widest and the furthest

@pytest.mark.parametrize("fan_in,fan_out", [(65536, 24), (24, 65536)])
def test_as_many_features_as_there_may_be(fan_in, fan_out):
    lengths, tail = [20, 0, 13], 1
    gen = torch.Generator().manual_seed(fan_in)
    rows, offsets = sum(lengths) + tail, [0] + np.cumsum(lengths).tolist()
    x, dz = (torch.randn(rows, n, generator=gen).to(BF16) for n in (fan_in, fan_out))
    w = (torch.randn(3, fan_out, fan_in, generator=gen) / math.sqrt(fan_in)).to(BF16)
    off = torch.tensor(offsets).cuda()
    ref.assert_near(binding.pcc_grouped_linear(x.cuda(), w.cuda(), None, off, ref.LEAKY), *ref.linear(x, w, None, offsets, ref.LEAKY), "y")
    got = binding.pcc_grouped_linear_grad(dz.cuda(), x.cuda(), w.cuda(), off, ref.RELU)
    for name, part, (value, bound) in zip(("dx", "dw", "db"), got, ref.linear_grad(dz, x, w, offsets, ref.RELU)):
        ref.assert_near(part, value, bound, name)


@pytest.mark.parametrize("rows,fan_in,fan_out", [(600, 200, 21900), (300, 200, 264), (300, 201, 264), (300, 160, 128)])
def test_rows_as_far_apart_as_they_may_be(rows, fan_in, fan_out):
    """2^22 elements: a row's place in a tile is 31 bits of bytes from the tile's first."""
    ld = 1 << 22
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dz = (torch.randn(rows, n, generator=gen, device="cuda").to(BF16) for n in (fan_in, fan_out))
    w, off = torch.randn(1, fan_out, fan_in, generator=gen, device="cuda").to(BF16), torch.tensor([0, rows], device="cuda")
    far = lambda n: torch.empty((rows, ld), dtype=BF16, device="cuda")[:, :n]  # noqa: E731
    x_far = far(fan_in)
    x_far.copy_(x)
    y = binding.pcc_grouped_linear(x_far, w, None, off, ref.RELU, out=far(fan_out))
    assert torch.equal(y, binding.pcc_grouped_linear(x, w, None, off, ref.RELU))
    del y
    if fan_out > 10000:
        return
    dz_far = far(fan_out)
    dz_far.copy_(dz)
    got, want = binding.pcc_grouped_linear_grad(dz_far, x_far, w, off, ref.RELU, dx=far(fan_in)), binding.pcc_grouped_linear_grad(dz, x, w, off, ref.RELU)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
