"""Arguments of the calls behind the router that contradict each other (no GPU needed)."""
import pytest
import torch

import paper_2607_22595_b200 as mix


def test_a_buffer_for_d_y_is_not_passed_over():
    x, i = torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="want_y"):
        mix.expert_combine_grad(x, x, x[:, :2], i, d_y=torch.zeros_like(x))
