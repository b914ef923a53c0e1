"""Launch chaining and tensor memory.  A chained successor may hold tensor memory while it waits for the end of its predecessor, so a
kernel lets its successor start only when it holds its own, and holds none while it waits itself."""
import os
import re

import pytest

from paper_2502_04416_b200 import build


def _kernels(name):
    """(kernel, its text) of a file, in the order of the file."""
    text = open(os.path.join(build.CSRC, name)).read()
    parts = re.split(r"__global__", text)[1:]
    return [(re.search(r"(\w+_kernel)\s*\(", p).group(1), p) for p in parts]


@pytest.mark.parametrize("kernel", ["adapter_umma_kernel", "adapter_outer_umma_kernel"])
def test_successors_start_after_the_allocation(kernel):
    body = dict(_kernels("adapters_umma.cuh"))[kernel]
    at = [body.index(f"{call}(") for call in ("grid_dep_wait", "tmem_alloc", "grid_dep_trigger")]
    assert at == sorted(at)
    assert "__syncthreads();" in body[at[1]:at[2]]           # one warp allocates, every thread lets go


@pytest.mark.gpu
@pytest.mark.parametrize("rows,r", [(1100, 64), (4200, 32)])
def test_layers_chained_to_adapters(rows, r):
    """Gradients on tcgen05 and layers whose routers allocate before they wait, one after another without a pause."""
    import torch
    from paper_2502_04416_b200 import binding, workloads as wl
    from tests import parity
    from tests.test_gpu_adapters import make
    inp = wl.make_inputs(wl.Workload("chained", wl.LayerShape(256, 1024, 8, 2, 2, "bf16"), (rows,), seed=3))
    layer = parity.gpu_layer(inp.layers[0], rows)
    x = parity.to_device(inp.x, "bf16")
    s = make("bf16", rows, 5, r, 256, 256, seed=1, dy=True)
    args = (s["a"], s["b"], s["ids"], s["scale"])
    want = layer.forward(x)
    want_a = layer.forward_adapted(x, *args)
    out, z = binding.adapter_forward(x, *args, want_z=True)
    grads = binding.adapter_backward(s["dy"], x, z, *args)
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        got.append((layer.forward_adapted(x, *args), layer.forward(x), *binding.adapter_backward(s["dy"], x, z, *args), layer.forward(x),
                    binding.adapter_forward(x, *args), layer.forward(x)))
    torch.cuda.synchronize()
    for g in got:
        for u, v in zip(g, (want_a, want, *grads, want, out, want)):
            assert torch.equal(u, v)
    assert layer.status() == 0 and binding.adapter_status() == 0
    layer.destroy()
