"""-m gpu: the sums over rows by the ring of bulk copies, at row counts around its depth: batches that end before the ring is full, just
as it is, and behind it, in blocks of their own (five adapters over 4096 + 4096 columns leave nothing to split) and in clusters."""
import numpy as np
import pytest

from paper_2502_04416_b200 import binding
from tests.test_gpu_adapters import check_backward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("r,steps", [(8, (1, 2, 3, 4, 7)), (16, (2, 3, 4)), (32, (3, 4, 5)), (64, (1, 2, 3))])
@pytest.mark.parametrize("n,d", [(5, 4096), (2, 72)])
def test_batches_around_the_depth_of_the_ring(r, steps, n, d):
    import torch
    for k in steps:
        for more in (0, 1):
            ids = np.random.default_rng(k).permutation(np.repeat(np.arange(n), 64 * k + more))
            rows = len(ids)
            s = make("bf16", rows, n, r, d, d, ids=None, dy=True)
            s["ids_np"], s["ids"] = ids, torch.from_numpy(ids.astype(np.int32)).cuda()
            args = (s["a"], s["b"], s["ids"], s["scale"])
            _, z = binding.adapter_forward(s["x"], *args, want_z=True)
            got = binding.adapter_backward(s["dy"], s["x"], z, *args, want_dx=False)
            if d < 100:
                check_backward(s, "bf16", got, z, dx_base=False)
            else:
                pick = [0, 7, 63, 64, 255, 256, 2049, 4095]              # the oracle on some columns of x, of dy all
                part = {**s, "x": s["x"][:, pick], "a": s["a"][:, :, pick]}
                check_backward(part, "bf16", (None, got[1][:, :, pick], None), z, dx_base=False)
                part = {**s, "dy": s["dy"][:, pick], "b": s["b"][:, pick]}
                check_backward(part, "bf16", (None, None, got[2][:, pick]), z, dx_base=False)
    assert binding.adapter_status() == 0
