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
