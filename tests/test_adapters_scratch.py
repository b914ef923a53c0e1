"""What the adapters' calls say about their scratch.  On the CPU nothing is launched: a call is refused for its scratch before the
device is asked for."""
import ctypes as C
import itertools

import pytest

from paper_2502_04416_b200 import binding, build

P = 1 << 20                                                 # an aligned address that nobody reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _ad(n, r, dtype):
    return binding.CmoeAdapters(n, r, 64, 32, dtype, P, P, None)


@pytest.mark.parametrize("with_ids,backward", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_scratch_never_shrinks_with_more_rows(lib, with_ids, backward):
    """Every row count around those where a batch changes its tiles."""
    for dtype, n, r in itertools.product((0, 1), (1, 5, 32, 64, 200), (8, 16, 24, 32, 40, 64)):
        ad = C.byref(_ad(n, r, dtype))
        for edge in {256, 1024, 4096, 32 * n, 64 * n}:
            sizes = [lib.cmoe_adapter_scratch_bytes(ad, rows, with_ids, backward) for rows in range(max(edge - 130, 1), edge + 131)]
            assert sizes == sorted(sizes), (dtype, n, r, edge)
        assert lib.cmoe_adapter_scratch_bytes(ad, 1 << 20, with_ids, backward) >= sizes[-1]


def test_a_small_scratch_is_named(lib):
    ad = _ad(4, 8, 0)
    need = lib.cmoe_adapter_scratch_bytes(C.byref(ad), 257, 1, 0)
    assert lib.cmoe_adapter_forward(C.byref(ad), None, 64, P, 257, None, None, 0, 1 << 40, 32, None, P, need, None) == -1
    assert b"scratch" not in lib.cmoe_last_error()          # another refusal's text is there
    assert lib.cmoe_adapter_forward(C.byref(ad), P, 64, P, 257, None, None, 0, 1 << 40, 32, None, P, need - 1, None) == -4
    assert b"scratch" in lib.cmoe_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("n,r,most", [(1, 24, 4096), (3, 64, 1024), (60, 32, 4100)])
def test_a_workspace_for_the_longest_batch_serves_shorter_ones(n, r, most):
    import torch
    g = torch.Generator("cuda").manual_seed(r)
    a, b = torch.randn(n, r, 64, generator=g, device="cuda").bfloat16(), torch.randn(n, 72, r, generator=g, device="cuda").bfloat16()
    room = [torch.empty(binding.adapter_scratch_bytes(n, r, 64, 72, torch.bfloat16, most, backward=k), dtype=torch.uint8, device="cuda") for k in (False, True)]
    for rows in (most, most - 1, most - 16, most - 100, 300):
        x, dy = torch.randn(rows, 64, generator=g, device="cuda").bfloat16(), torch.randn(rows, 72, generator=g, device="cuda").bfloat16()
        ids = torch.randint(-1, n, (rows,), generator=g, device="cuda").to(torch.int32)
        out, z = binding.adapter_forward(x, a, b, ids, want_z=True, scratch=room[0])
        want, want_z = binding.adapter_forward(x, a, b, ids, want_z=True)
        assert torch.equal(out, want) and torch.equal(z, want_z)
        for u, v in zip(binding.adapter_backward(dy, x, z, a, b, ids, scratch=room[1]), binding.adapter_backward(dy, x, z, a, b, ids)):
            assert torch.equal(u, v)
