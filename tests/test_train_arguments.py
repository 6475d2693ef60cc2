"""More calls that the training operators refuse, before anything touches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2212_01185_amd import binding, synth, train


@pytest.mark.parametrize("eps", [1e-40, -1e-8, float("nan")])
def test_adamw_wants_an_eps_with_a_reciprocal(eps):
    with pytest.raises(ValueError, match="eps"):
        binding.AdamW([torch.zeros(3)], [torch.zeros(3)], eps=eps)


@pytest.mark.parametrize("eps", [0.0, float("nan")])
def test_trainer_wants_an_eps(eps):
    """The weights of padded inputs have gradients of 0 in every step: 0 / (0 + 0), and with them every output, would be NaN."""
    with pytest.raises(ValueError, match="eps"):
        train.Trainer(synth.make_blob(0), eps=eps)


PARAM, GRAD, COPY, M, V = (0x10000 * i for i in range(1, 6))       # stand for device pointers: a refused call never follows them


@pytest.mark.parametrize("grad_type,grad", [(2, M), (2, V + 396), (2, PARAM - 396), (2, PARAM + 4), (0, PARAM), (0, COPY), (2, COPY - 4), (0, M + 398)])
def test_adamw_refuses_a_gradient_where_it_writes(grad_type, grad):
    """Another wave may have written an element before its gradient is read."""
    t = (binding._AdamwTensor * 2)()
    t[0] = binding._AdamwTensor(PARAM, grad, COPY, M, V, None, None, 100)
    t[1] = binding._AdamwTensor(PARAM + 0x1000, GRAD, None, M + 0x1000, V + 0x1000, None, None, 100)
    h = C.c_void_p()
    assert binding.load().pcc_adamw_create(C.byref(h), t, 2, grad_type, 0, 32, 0) == binding.PCC_E_ARG


def test_operators_that_autograd_does_not_record_refuse_its_tensors():
    """A result without a graph would drop the gradients of everything before it, and say nothing."""
    t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    asks = lambda x: x.requires_grad_(True)  # noqa: E731
    off, f = torch.tensor([0, 4]), torch.zeros(4, 60)
    rgb = torch.zeros(4, 3, dtype=torch.uint8)
    calls = (lambda: binding.pcc_grouped_linear(asks(t(4, 8)), t(1, 3, 8), None, off),
             lambda: binding.pcc_grouped_linear(t(4, 8), asks(t(1, 3, 8)), None, off),
             lambda: binding.pcc_grouped_linear(t(4, 8), t(1, 3, 8), asks(torch.zeros(1, 3)), off),
             lambda: binding.pcc_grouped_linear(t(4, 8), t(1, 3, 8), None, off, out=asks(t(4, 3))),
             lambda: binding.pcc_grouped_linear_grad(asks(t(4, 3)), t(4, 8), t(1, 3, 8), off),
             lambda: binding.pcc_grouped_linear_grad(t(4, 3), asks(t(4, 8)), t(1, 3, 8), off),
             lambda: binding.pcc_grouped_linear_grad(t(4, 3), t(4, 8), asks(t(1, 3, 8)), off),
             lambda: binding.pcc_mixture_loss(asks(f.clone()), rgb),
             lambda: binding.pcc_mixture_loss(f, rgb, weight=asks(torch.ones(4))))
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):        # off: the next check, that tensors are on a GPU
            call()


def _refused(name, defaults, **changes):
    args = dict(defaults)
    assert set(changes) <= set(args)
    args.update(changes)
    return getattr(binding.load(), name)(*args.values()) == binding.PCC_E_ARG


A, B, D, E, F, G, H = (0x100000 * i for i in range(1, 8))
CONTEXTS = dict(img=A, n=2, H=16, W=8, nbhd=10, delay=2, x=B, width=32, ldx=32, stream=None)
LINEAR = dict(x=A, ldx=32, w=B, bias=D, off=E, groups=2, rows=100, fan_in=32, fan_out=16, type=0, act=0, y=F, y_type=0, ldy=16, stream=None)
BACKWARD = dict(dz=A, lddz=16, x=B, ldx=32, w=D, off=E, groups=2, rows=100, fan_in=32, fan_out=16, type=0, x_act=0, dx=F, lddx=32, dw=G, db=H,
                workspace=0x900000, workspace_bytes=1 << 20, stream=None)
LOSS = dict(params=A, ldp=60, rgb=B, weight=D, count=100, K=5, dist=0, scale=1.0, bits=E, grad=F, grad_type=2, ldg=60, stream=None)


@pytest.mark.parametrize("name,defaults,changes", [
    ("pcc_contexts", CONTEXTS, dict(x=A)), ("pcc_contexts", CONTEXTS, dict(x=A + 3 * 256 - 2)), ("pcc_contexts", CONTEXTS, dict(x=A - 2 * 32 * 256 + 2)),
    ("pcc_grouped_linear", LINEAR, dict(y=A)), ("pcc_grouped_linear", LINEAR, dict(y=A + 2 * 3199)), ("pcc_grouped_linear", LINEAR, dict(y=B + 2046)),
    ("pcc_grouped_linear", LINEAR, dict(y=D + 126)), ("pcc_grouped_linear", LINEAR, dict(y=E + 22)), ("pcc_grouped_linear", LINEAR, dict(y=A - 3198)),
    ("pcc_grouped_linear", LINEAR, dict(y=A - 6396, y_type=2)),
    # columns of one buffer that run into each other: to the right, and into the next row
    ("pcc_grouped_linear", LINEAR, dict(ldx=48, ldy=48, y=A + 62)), ("pcc_grouped_linear", LINEAR, dict(ldx=47, ldy=47, y=A + 64)),
    ("pcc_grouped_linear", LINEAR, dict(ldx=47, ldy=47, y=A - 30)), ("pcc_grouped_linear", LINEAR, dict(ldx=48, ldy=49, y=A + 64)),
    ("pcc_grouped_linear_grad", BACKWARD, dict(dx=A)), ("pcc_grouped_linear_grad", BACKWARD, dict(dx=B)), ("pcc_grouped_linear_grad", BACKWARD, dict(dx=D)),
    ("pcc_grouped_linear_grad", BACKWARD, dict(dx=E)), ("pcc_grouped_linear_grad", BACKWARD, dict(dx=G)), ("pcc_grouped_linear_grad", BACKWARD, dict(dx=H)),
    ("pcc_grouped_linear_grad", BACKWARD, dict(dw=A)), ("pcc_grouped_linear_grad", BACKWARD, dict(dw=B)), ("pcc_grouped_linear_grad", BACKWARD, dict(dw=D)),
    ("pcc_grouped_linear_grad", BACKWARD, dict(dw=E)), ("pcc_grouped_linear_grad", BACKWARD, dict(db=A)), ("pcc_grouped_linear_grad", BACKWARD, dict(db=B)),
    ("pcc_grouped_linear_grad", BACKWARD, dict(db=D)), ("pcc_grouped_linear_grad", BACKWARD, dict(db=E)), ("pcc_grouped_linear_grad", BACKWARD, dict(db=G + 4092)),
    ("pcc_mixture_loss", LOSS, dict(grad=A + 4)), ("pcc_mixture_loss", LOSS, dict(grad=A, ldg=61)), ("pcc_mixture_loss", LOSS, dict(grad=A, grad_type=0)),
    ("pcc_mixture_loss", LOSS, dict(grad=B)), ("pcc_mixture_loss", LOSS, dict(grad=D)), ("pcc_mixture_loss", LOSS, dict(bits=A)),
    ("pcc_mixture_loss", LOSS, dict(bits=B)), ("pcc_mixture_loss", LOSS, dict(bits=D)), ("pcc_mixture_loss", LOSS, dict(bits=F)),
    ("pcc_mixture_loss", LOSS, dict(ldp=120, ldg=120, grad=A + 236))])
def test_outputs_that_overlap_are_refused(name, defaults, changes):
    """What is written first would be read, or written over."""
    assert _refused(name, defaults, **changes)


@pytest.mark.parametrize("space", [A, B, D, E, F, G, H])
def test_a_workspace_that_overlaps_is_refused(space):
    rows, far = 40000, 0x10000000
    need = binding.load().pcc_grouped_linear_grad_workspace_bytes(rows, 2, 32, 16)
    assert 0 < need < far
    args = {k: v * 0x100 if v in (A, B, D, E, F, G, H) else v for k, v in BACKWARD.items()}
    assert _refused("pcc_grouped_linear_grad", args, rows=rows, workspace=space * 0x100 - need + 16, workspace_bytes=need)


@pytest.mark.parametrize("name,defaults,changes", [
    ("pcc_contexts", CONTEXTS, dict(n=3, H=1 << 15, W=1 << 16, x=1 << 40)), ("pcc_grouped_linear", LINEAR, dict(rows=1 << 32, fan_in=7, fan_out=5, y=1 << 60)),
    ("pcc_grouped_linear_grad", BACKWARD, dict(rows=1 << 32, fan_in=7, fan_out=5, dz=1 << 50, x=1 << 52, dx=1 << 54, workspace=1 << 56, workspace_bytes=1 << 40)),
    ("pcc_mixture_loss", LOSS, dict(count=1 << 33, params=1 << 50, rgb=1 << 52, weight=1 << 53, bits=1 << 54, grad=1 << 56))])
def test_more_threads_than_a_launch_has_are_refused(name, defaults, changes):
    assert _refused(name, defaults, **changes)
