"""Optimizer states of a training step where blocks, networks and numbers meet their limits.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2212_01185_amd import binding, synth, train

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.contiguous().view(torch.uint8)


def _fill(trainer, step, dirty=None):
    """Gradients of every network, of very different sizes; `dirty`: (network, value) of one element of each bias."""
    gen = torch.Generator().manual_seed(step)
    for t in trainer.dw + trainer.db:
        for g in range(trainer.groups):
            t[g] = (torch.randn(t[g].shape, generator=gen) * 10.0 ** (2 * g - 3)).to(t.device)
    if dirty:
        for t in trainer.db:
            t[dirty[0], 5] = dirty[1]


@pytest.mark.parametrize("state_bits", [32, 8])
@pytest.mark.parametrize("make", [synth.make_blob, synth.make_paper_blob])
def test_a_network_moves_as_it_would_alone(make, state_bits):
    """From the same gradients, whatever the other networks' are: the same bits, also where one of the others' moments is not finite."""
    blobs = [make(s) for s in (1, 2, 3)]
    hyper = dict(lr=1e-3, weight_decay=0.01, state_bits=state_bits)
    together, alone = train.Trainer(blobs, **hyper), [train.Trainer(b, **hyper) for b in blobs]
    for step in range(4):
        _fill(together, step, (1, float("inf")) if step == 2 else None)
        for g, one in enumerate(alone):
            for mine, all_of in zip(one.dw + one.db, together.dw + together.db):
                mine.copy_(all_of[g:g + 1])
            one.optimizer.pcc_adamw_step()
        together.optimizer.pcc_adamw_step()
        for g, one in enumerate(alone):
            for name in ("w", "b", "w16"):
                for i, (a, b) in enumerate(zip(getattr(one, name), getattr(together, name))):
                    assert torch.equal(_bits(a), _bits(b[g:g + 1])), (step, g, name, i)
    for g in (0, 2):
        assert all(torch.isfinite(t[g]).all() for t in together.w + together.b)


@pytest.mark.parametrize("state_bits", [32, 8])
def test_a_step_goes_down_its_gradient(state_bits):
    """Trainer.step moves weights by the AdamW step of the gradients that it leaves."""
    hyper = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
    trainer = train.Trainer([synth.make_blob(1), synth.make_blob(2)], state_bits=state_bits, **hyper)
    before = [t.cpu().numpy() for t in trainer.w + trainer.b]
    img = synth.make_image(3, synth.ImageSpec(33, 20, 5, 4.0, 20.0))
    d = torch.from_numpy(np.stack([img])).cuda()
    trainer.step([d, d])
    for i, (p, now, g) in enumerate(zip(before, trainer.w + trainer.b, trainer.dw + trainer.db)):
        one = ref.AdamW(p.reshape(-1), 32, **hyper)         # the update uses the moments before they are rounded
        one.step(g.cpu().numpy().reshape(-1))
        # a quotient of at most 1 from some ten roundings on each side, times the rate; the parameter's product and difference on each side
        tol = 2.0 ** -24 * (24 * hyper["lr"] + 4 * np.abs(one.p))
        assert np.all(np.abs(now.cpu().numpy().reshape(-1) - one.p) <= tol), i
        assert np.any(now.cpu().numpy() != p)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 3e30])
def test_a_moment_that_is_not_finite_stays_in_its_element(grad_dtype, value):
    """In 8 bits as in 32: the others of its block have the states and parameters that they have where its gradient is 0."""
    if grad_dtype == torch.float16 and value == 3e30:
        pytest.skip("no such number")
    n, at = 1024, 300
    gen = torch.Generator().manual_seed(7)
    start = torch.randn(n, generator=gen).cuda()
    values = [torch.randn(n, generator=gen).to(grad_dtype) for _ in range(4)]

    def run(dirty, bits):
        p, g = [start.clone()], [torch.zeros(n, dtype=grad_dtype, device="cuda")]
        opt = binding.AdamW(p, g, state_bits=bits)
        out = []
        for k, v in enumerate(values):
            g[0].copy_(v)
            g[0][at] = dirty if k == 1 else 0.0
            opt.pcc_adamw_step()
            scales = [opt.m_scale[0].clone(), opt.v_scale[0].clone()] if bits == 8 else []
            out.append([p[0].clone(), _bits(opt.m[0]).clone().view(n, -1), _bits(opt.v[0]).clone().view(n, -1)] + scales)
        return out

    others = torch.arange(n, device="cuda") != at
    for bits in (32, 8):
        clean, dirty = run(0.0, bits), run(value, bits)
        for k, (a, b) in enumerate(zip(clean, dirty)):
            if value == 3e30 and bits == 8:                 # the first moment is finite, and its block's scale is its own
                a, b = [a[0][~block(at, n)], a[2], a[4]], [b[0][~block(at, n)], b[2], b[4]]
                assert torch.equal(a[0], b[0]) and torch.equal(a[1][others], b[1][others]) and torch.equal(a[2], b[2]), (bits, k)
                continue
            for x, y in zip(a[:3], b[:3]):
                assert torch.equal(x[others], y[others]), (bits, k)
            assert all(torch.equal(x, y) for x, y in zip(a[3:], b[3:])), (bits, k)
        assert value == 3e30 or torch.isnan(dirty[-1][0][at])


def block(at, n):
    i = torch.arange(n, device="cuda")
    return i // binding.STATE_BLOCK == at // binding.STATE_BLOCK


def test_an_eps_below_the_normal_numbers_is_refused():
    """Its reciprocal would be infinite: an element without any gradient became NaN."""
    p, g = [torch.ones(64, device="cuda")], [torch.zeros(64, device="cuda")]
    opt = binding.AdamW(p, g, lr=0.5, weight_decay=0.0)
    for eps in (1e-40, -1e-8, float("nan")):
        opt.eps = eps
        with pytest.raises(binding.PccError) as e:
            opt.pcc_adamw_step()
        assert e.value.code == binding.PCC_E_ARG
    opt.eps = 2.0 ** -126
    opt.pcc_adamw_step()
    assert (p[0] == 1).all() and opt.step.item() == 1


def test_pictures_without_pixels():
    """Tensors of no pictures count as none, and every network's being one is refused as no pictures are."""
    trainer = train.Trainer([synth.make_blob(1), synth.make_blob(2)])
    d = torch.randint(0, 256, (2, 9, 7, 3), dtype=torch.uint8, device="cuda")
    want = trainer.gradients([d, []]).clone()
    dw = [t.clone() for t in trainer.dw]
    got = trainer.gradients([[d[:0], d], d[:0]])
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(dw, trainer.dw))
    with pytest.raises(ValueError, match="pictures"):
        trainer.gradients([d[:0], [d[:, :0]]])


def test_gradients_that_touch_or_share_memory():
    """Gradients right beside what is written, one gradient of two parameters, and a gradient that is its parameter."""
    space = torch.randn(600, device="cuda")
    p, q, g = space[:200], space[400:], space[200:400]
    start = [t.clone() for t in (p, q, g)]
    binding.AdamW([p, q], [g, g]).pcc_adamw_step()
    for t, before in ((p, start[0]), (q, start[1])):
        alone = before.clone()
        binding.AdamW([alone], [start[2].clone()]).pcc_adamw_step()
        assert torch.equal(t, alone)
    assert torch.equal(g, start[2])
    own, apart = start[0].clone(), start[0].clone()
    binding.AdamW([own], [own]).pcc_adamw_step()
    binding.AdamW([apart], [start[0].clone()]).pcc_adamw_step()
    assert torch.equal(own, apart)
    with pytest.raises(binding.PccError):
        binding.AdamW([p, q], [g, p])


def test_parameters_of_a_module_without_autograd():
    """What requires gradients is taken where autograd is off, and always by the optimizer, which writes in place."""
    x, off = torch.randn(5, 8, device="cuda").bfloat16(), torch.tensor([0, 5], device="cuda")
    w = torch.nn.Parameter(torch.randn(1, 3, 8, device="cuda"))
    w16 = torch.nn.Parameter(w.detach().bfloat16())
    with torch.no_grad():
        y = binding.pcc_grouped_linear(x, w16, None, off)
        _, dw, _ = binding.pcc_grouped_linear_grad(y, x, w16, off, want_dx=False)
    assert torch.equal(y, binding.pcc_grouped_linear(x, w16.detach(), None, off))
    before = w.detach().clone()
    binding.AdamW([w], [dw]).pcc_adamw_step()
    assert not torch.equal(before, w.detach())


def test_outputs_beside_their_inputs_in_one_buffer():
    """Columns of one buffer, and rows that end where others begin, are no overlap."""
    rows, off = 70, torch.tensor([0, 70], device="cuda")
    gen = torch.Generator().manual_seed(4)
    x0, w = torch.randn(rows, 32, generator=gen).bfloat16().cuda(), torch.randn(1, 16, 32, generator=gen).bfloat16().cuda()
    dz0, bias = torch.randn(rows, 16, generator=gen).bfloat16().cuda(), torch.zeros(1, 16, device="cuda")
    want = binding.pcc_grouped_linear(x0, w, bias, off)
    dx0, dw0, db0 = binding.pcc_grouped_linear_grad(dz0, x0, w, off)
    for first in (0, 16):                            # y in front of x, and behind it
        buffer = torch.zeros(rows, 48, device="cuda", dtype=torch.bfloat16)
        x, y = buffer[:, 16 - first:48 - first], buffer[:, 32:] if first else buffer[:, :16]
        x.copy_(x0)
        binding.pcc_grouped_linear(x, w, bias, off, out=y)
        assert torch.equal(y, want) and torch.equal(x, x0)
    buffer = torch.zeros(rows, 80, device="cuda", dtype=torch.bfloat16)
    dz, x, dx = buffer[:, :16], buffer[:, 16:48], buffer[:, 48:]
    dz.copy_(dz0)
    x.copy_(x0)
    _, dw, db = binding.pcc_grouped_linear_grad(dz, x, w, off, dx=dx)
    assert torch.equal(dx, dx0) and torch.equal(dw, dw0) and torch.equal(db, db0) and torch.equal(x, x0) and torch.equal(dz, dz0)
    line = torch.zeros(rows * 48, device="cuda", dtype=torch.bfloat16)
    x, y = line[:rows * 32].view(rows, 32), line[rows * 32:].view(rows, 16)
    x.copy_(x0)
    binding.pcc_grouped_linear(x, w, bias, off, out=y)
    assert torch.equal(y, want)
    params = torch.randn(rows, 120, generator=gen).cuda()
    rgb = torch.randint(0, 256, (rows, 3), generator=gen).to(torch.uint8).cuda()
    apart = binding.pcc_mixture_loss(params[:, :60].contiguous(), rgb)
    bits, grad = binding.pcc_mixture_loss(params[:, :60], rgb, grad=params[:, 60:])
    assert torch.equal(bits, apart[0]) and torch.equal(grad, apart[1])
