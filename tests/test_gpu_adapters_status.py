"""-m gpu: what the adapters' calls say after a bounded wait has run out, and of a layer on another device."""
import pytest

from paper_2502_04416_b200 import binding
from tests.test_gpu_adapters import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


def test_wait_timeout_is_reported_once_and_calls_go_on():
    """A wait that nothing ends runs to its (millisecond) limit on another stream, the kernel returns normally, the status reports its code
    once, and every form of the calls then computes right results."""
    import ctypes as C
    import torch
    assert binding.adapter_status() == 0
    side = torch.cuda.Stream()
    binding.adapter_selftest_wait_timeout(2_000_000, stream=side)
    torch.cuda.synchronize()
    w = C.c_int32()
    assert binding.load().cmoe_adapter_status(C.byref(w), binding._stream_ptr(None)) == -6      # CMOE_ERR_DEVICE_TIMEOUT
    assert w.value == 1 and b"wait" in binding.load().cmoe_last_error()
    assert binding.adapter_status() == 0                                                        # reported once, then cleared
    for dtype, rows, r in (("bf16", 20, 8), ("bf16", 300, 16), ("bf16", 1100, 64), ("bf16", 4100, 24), ("fp32", 300, 8)):
        s = make(dtype, rows, 3, r, 72, 136, dy=True)
        args = (s["a"], s["b"], s["ids"], s["scale"])
        out, z = binding.adapter_forward(s["x"], *args, base=s["base"], want_z=True)
        check_forward(s, dtype, out, z)
        check_backward(s, dtype, binding.adapter_backward(s["dy"], s["x"], z, *args, dx_base=s["dx_base"]), z)
    binding.adapter_selftest_wait_timeout(2_000_000)
    assert binding.adapter_status() == 1 and binding.adapter_status() == 0
    for limit in (10, 2_000_000_001):
        with pytest.raises(binding.CmoeError):
            binding.adapter_selftest_wait_timeout(limit)


def test_a_layer_on_another_device_is_refused():
    import torch
    from paper_2502_04416_b200 import workloads as wl
    from tests import parity
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    inp = wl.make_inputs(wl.Workload("elsewhere", wl.LayerShape(256, 1024, 8, 2, 2, "bf16"), (40,), seed=3))
    layer = parity.gpu_layer(inp.layers[0], 40)
    x = parity.to_device(inp.x, "bf16").to("cuda:1")
    a, b = torch.zeros(1, 8, 256, dtype=torch.bfloat16, device="cuda:1"), torch.zeros(1, 256, 8, dtype=torch.bfloat16, device="cuda:1")
    with pytest.raises(binding.CmoeError, match="another device"):
        layer.forward_adapted(x, a, b)
    layer.destroy()
