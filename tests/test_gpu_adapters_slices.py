"""-m gpu: slices of a set of adapters as sets of their own."""
import pytest

from paper_2502_04416_b200 import binding
from tests.test_gpu_adapters import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [40, 400])
def test_a_slice_of_a_set_of_adapters(dtype, rows):
    """a[k:], b[k:] and scale[k:] are a set of adapters for every k, on whatever boundary the scales then start.  Against the oracle, not
    the whole set's results: how many blocks share a sum goes by the number of adapters, and with it the order of the terms."""
    for k in (1, 2, 3):
        s = make(dtype, rows, 5, 8, 64, 96, seed=k, dy=True)
        whole = dict(s)
        s["ids"] = whole["ids"].where(whole["ids"] < k, whole["ids"] - k).where(whole["ids"] >= k, whole["ids"].new_full((), -1))
        s["ids_np"] = s["ids"].cpu().numpy()
        s["a"], s["b"], s["scale"] = (whole[name][k:] for name in ("a", "b", "scale"))
        assert s["scale"].data_ptr() == whole["scale"].data_ptr() + 4 * k
        out, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=s["base"], want_z=True)
        check_forward(s, dtype, out, z)
        got = binding.adapter_backward(s["dy"], s["x"], z, s["a"], s["b"], s["ids"], s["scale"], dx_base=s["dx_base"])
        check_backward(s, dtype, got, z)


def test_a_slice_beside_a_layer_and_in_a_graph():
    """The same for the call beside a layer, captured and replayed after the scales have changed."""
    import torch
    from paper_2502_04416_b200 import workloads as wl
    from tests import parity
    inp = wl.make_inputs(wl.Workload("slice", wl.LayerShape(256, 1024, 8, 2, 2, "bf16"), (40,), seed=3))
    layer = parity.gpu_layer(inp.layers[0], 40)
    x = parity.to_device(inp.x, "bf16")
    g = torch.Generator("cuda").manual_seed(1)
    a, b = torch.randn(4, 8, 256, generator=g, device="cuda").bfloat16(), torch.randn(4, 256, 8, generator=g, device="cuda").bfloat16()
    scale, ids = torch.rand(4, generator=g, device="cuda"), (torch.arange(40, device="cuda") % 3).to(torch.int32)
    want = layer.forward_adapted(x, a, b, ids + 1, scale)
    assert torch.equal(layer.forward_adapted(x, a[1:], b[1:], ids, scale[1:]), want)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward_adapted(x, a[1:], b[1:], ids, scale[1:], out=out)
    for f in (1.0, 2.0):
        scale.mul_(f)
        want = layer.forward_adapted(x, a, b, ids + 1, scale)
        out.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    layer.destroy()
