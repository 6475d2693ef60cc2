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
