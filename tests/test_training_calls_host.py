"""CPU checks of the Python side of the training calls: what it refuses before any GPU work, how it
is built and what the package does without it."""
import pytest
import torch


def test_a_checkpoint_to_save_to_needs_a_save():
    """It used to be left as it was, in silence."""
    from paper_2108_08842_b200 import _binding

    native = _binding.native(0, 0, 0, 0, 0, 1)
    x, w = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(8, 32, dtype=torch.bfloat16)
    saved = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8)
    with pytest.raises(ValueError, match="saved is given"):
        _binding.linear(native, x, w, None, "none", None, None, "none", saved)
