"""-m gpu: sizes at the ends of what the calls take."""
import numpy as np
import pytest

from oracle import adapters_oracle as ao
from paper_2502_04416_b200 import binding
from paper_2502_04416_b200.binding import Dropout

pytestmark = pytest.mark.gpu


def test_counts_past_32_bits_are_refused():
    """A row of 2^32 + 5 columns is not one of five."""
    import torch
    x = torch.empty(1, 2**32 + 5, dtype=torch.bfloat16, device="cuda")
    for t in (x, x.view(-1, 1), x[:, :2**31], x.view(-1, 1)[:2**31]):
        with pytest.raises(ValueError):
            binding.dropout(t, Dropout(0.5), out=t)
    a, b = torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, 8, dtype=torch.bfloat16, device="cuda")
    wide = b.expand(1, 2**32 + 64, 8)                                        # no memory behind it
    with pytest.raises(ValueError, match="dimension"):
        binding.adapter_forward(x[:, :64], a, wide)
    with pytest.raises(ValueError, match="rows or columns"):
        binding.adapter_forward(x.view(-1, 1)[:2**31], a, b)
    with pytest.raises(ValueError, match="rows or columns"):
        binding.adapter_backward(x, x, None, a, b)
