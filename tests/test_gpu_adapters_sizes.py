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


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("first", [0, 1])
def test_the_widest_row(dtype, first):
    """2^31 - 1 columns, on a 16-byte boundary and off it, in place: the first and the last of them against the oracle's mask, and the
    elements beside the row untouched."""
    import torch
    cols = 2**31 - 1
    buf = torch.ones(cols + 2, dtype=getattr(torch, dtype), device="cuda")
    x = buf[first:first + cols].view(1, cols)
    drop = Dropout(0.5, 2**40 + 3, 9, 2**32 - 1)
    binding.dropout(x, drop, out=x)
    blocks = np.concatenate([np.arange(4), cols // 8 - 3 + np.arange(4)])
    c = np.zeros((len(blocks), 4), dtype=np.uint32)
    c[:, 0], c[:, 1], c[:, 2] = blocks, 2**32 - 1, 9
    words = ao.philox(c, ((2**40 + 3) % 2**32, (2**40 + 3) >> 32))
    keep = np.stack([words & 0xFFFF, words >> 16], axis=-1).reshape(-1) >= ao.threshold(0.5)
    at = (blocks[:, None] * 8 + np.arange(8)).reshape(-1)
    keep, at = keep[at < cols], at[at < cols]
    assert at[-1] == cols - 1
    got = x[0, torch.from_numpy(at).cuda()].double().cpu().numpy()
    np.testing.assert_array_equal(got, np.where(keep, 2.0, 0.0))
    assert (buf[:first] == 1).all() and (buf[first + cols:] == 1).all()
    counts = [(x[0, i:i + 2**28] == 2).sum() for i in range(0, cols, 2**28)]
    kept = int(torch.stack(counts).sum())
    assert abs(kept - cols / 2) < 6 * (cols / 4) ** 0.5                      # binomial: six standard deviations
