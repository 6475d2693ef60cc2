"""More calls that the training operators refuse, before anything touches a GPU."""
import pytest
import torch

from paper_2212_01185_amd import binding


@pytest.mark.parametrize("eps", [1e-40, -1e-8, float("nan")])
def test_adamw_wants_an_eps_with_a_reciprocal(eps):
    with pytest.raises(ValueError, match="eps"):
        binding.AdamW([torch.zeros(3)], [torch.zeros(3)], eps=eps)
