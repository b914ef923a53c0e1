"""-m gpu: calls of several host threads, each on its own stream with its own buffers."""
import ctypes as C
import threading

import pytest

from paper_2502_04416_b200 import binding

pytestmark = pytest.mark.gpu


def _loop(calls, turns, go, bad):
    """Every call `turns` times over; the statuses that were not 0."""
    go.wait()
    for _ in range(turns):
        for call in calls:
            st = call()
            if st:
                bad.append((st, binding.load().cmoe_last_error()))


def _in_threads(jobs, turns):
    go, bad = threading.Barrier(len(jobs)), []
    threads = [threading.Thread(target=_loop, args=(j, turns, go, bad)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return bad


@pytest.mark.parametrize("what", ["cluster of the products", "adapters of the sort"])
def test_launches_of_one_kernel_with_different_shared_memory(what):
    """Two threads launch the same kernels, which need different amounts of shared memory for different calls: fp32 products of one
    tile take eight blocks a cluster, those of 40 tiles four; the sort's tables grow with the number of adapters."""
    import torch
    lib = binding.load()
    if what == "cluster of the products":
        shapes = [(20, 1, False), (1280, 1, False)]
        dtype, d = torch.float32, 4096
    else:
        shapes = [(300, 1024, True), (300, 330, True)]
        dtype, d = torch.bfloat16, 64
    jobs, keep = [], []
    for i, (rows, n, with_ids) in enumerate(shapes):
        g = torch.Generator("cuda").manual_seed(i)
        x = torch.randn(rows, d, generator=g, device="cuda").to(dtype)
        a, b = torch.randn(n, 8, d, generator=g, device="cuda").to(dtype), torch.randn(n, d, 8, generator=g, device="cuda").to(dtype)
        ids = torch.randint(0, n, (rows,), generator=g, device="cuda").to(torch.int32) if with_ids else None
        out, want = torch.empty_like(x), binding.adapter_forward(x, a, b, ids)
        scratch = torch.empty(max(binding.adapter_scratch_bytes(n, 8, d, d, dtype, rows, with_ids), 1), dtype=torch.uint8, device="cuda")
        ad = binding.CmoeAdapters(n, 8, d, d, binding._dtype_code(x), a.data_ptr(), b.data_ptr(), None)
        stream = torch.cuda.Stream()
        keep.append((x, a, b, ids, out, want, scratch, ad, stream))
        args = (C.byref(ad), x.data_ptr(), d, ids.data_ptr() if with_ids else None, rows, None, None, 0, out.data_ptr(), d, None,
                scratch.data_ptr(), scratch.numel(), C.c_void_p(stream.cuda_stream))
        jobs.append([lambda args=args: lib.cmoe_adapter_forward(*args)])
    torch.cuda.synchronize()
    bad = _in_threads(jobs * 2, 3000)           # two threads of either kind; those of a kind write the same values
    torch.cuda.synchronize()
    assert not bad, (len(bad), bad[0])
    for _, _, _, _, out, want, *_ in keep:
        assert torch.equal(out, want)
