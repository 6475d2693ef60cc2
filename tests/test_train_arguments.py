"""More calls that the training operators refuse, before anything touches a GPU."""
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
