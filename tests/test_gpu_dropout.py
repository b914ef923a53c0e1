"""-m gpu: counter-based dropout (cmoe_dropout) against the 64-bit oracle: mask bit for bit, sums to one rounding."""
import numpy as np
import pytest

from oracle import adapters_oracle as ao
from paper_2502_04416_b200 import binding
from paper_2502_04416_b200.binding import Dropout

pytestmark = pytest.mark.gpu

DT = {"bf16": "bfloat16", "fp32": "float32"}


def _dtype(name):
    import torch
    return getattr(torch, DT[name])


def _rand(shape, dtype, seed):
    import torch
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(_dtype(dtype))


def _host(t):
    return t.double().cpu().numpy()


def _check(got, want, mag, dtype):
    """One rounding to the type (half a step: eps / 2) of a value whose fp32 arithmetic (the scale's rounding, the product and the
    sum: three roundings) is off by at most 4 * 2^-24 of the terms' magnitudes."""
    import torch
    eps = torch.finfo(_dtype(dtype)).eps
    bound = eps / 2 * np.abs(want) + 4 * 2.0**-24 * (1 + eps) * mag
    assert (np.abs(_host(got) - want) <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (2, 9), (77, 250), (129, 255), (64, 256), (5, 4096), (1000, 1377), (1, 100003)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 65535 / 65536])
def test_dropout_matches_definition(dtype, rows, cols, p):
    seed, offset, row0 = 2**63 + 12345, 2**33 + 7, 2**32 - rows
    x, r = _rand((rows, cols), dtype, 1), _rand((rows, cols), dtype, 2)
    inv = 65536 / (65536 - ao.threshold(p))
    drop = Dropout(p, seed, offset, row0)
    keep = ao.keep_mask(rows, cols, p, seed, offset, row0)
    got = binding.dropout(x, drop)
    np.testing.assert_array_equal(_host(got) != 0, keep & (_host(x) != 0))
    _check(got, ao.dropout(_host(x), p, seed, offset, row0), np.abs(_host(x)) * inv, dtype)
    got = binding.dropout(x, drop, residual=r)
    _check(got, ao.dropout(_host(x), p, seed, offset, row0, _host(r)), np.abs(_host(x)) * inv + np.abs(_host(r)), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols,ld,first", [(24, 40, 8), (24, 40, 3), (21, 40, 8), (21, 33, 1), (256, 264, 0)])
def test_strided_views_and_what_lies_between(dtype, cols, ld, first):
    import torch
    rows = 37
    wide_x, wide_r, wide_o = (_rand((rows + 1, ld + first), dtype, s) for s in (1, 2, 3))
    view = [t[:rows, first:first + cols] for t in (wide_x, wide_r, wide_o)]
    before = wide_o.clone()
    want = ao.dropout(_host(view[0]), 0.2, 5, residual=_host(view[1]))
    binding.dropout(view[0], Dropout(0.2, 5), residual=view[1], out=view[2])
    _check(view[2], want, np.abs(_host(view[0])) * 1.25001 + np.abs(_host(view[1])), dtype)
    wide_o[:rows, first:first + cols] = before[:rows, first:first + cols]
    assert torch.equal(wide_o, before)                                      # nothing outside the matrix was written


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [64, 61])
def test_in_place_and_parts(dtype, cols):
    import torch
    x, r = _rand((50, cols), dtype, 1), _rand((50, cols), dtype, 2)
    want = binding.dropout(x, Dropout(0.3, 9, 4), residual=r)
    a = x.clone()
    assert binding.dropout(a, Dropout(0.3, 9, 4), residual=r, out=a) is a and torch.equal(a, want)
    a = r.clone()
    binding.dropout(x, Dropout(0.3, 9, 4), residual=a, out=a)
    assert torch.equal(a, want)
    parts = [binding.dropout(x[i:j], Dropout(0.3, 9, 4, row0=i), residual=r[i:j]) for i, j in ((0, 1), (1, 33), (33, 50))]
    assert torch.equal(torch.cat(parts), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [64, 61])
def test_dropped_places_may_hold_anything(dtype, cols):
    import torch
    x, r = _rand((33, cols), dtype, 1), _rand((33, cols), dtype, 2)
    keep = torch.from_numpy(ao.keep_mask(33, cols, 0.4, 3)).cuda()
    bad = x.clone()
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"), torch.finfo(x.dtype).min)):
        bad.view(-1)[i::4] = v
    bad = torch.where(keep, x, bad)
    for res in (None, r):
        assert torch.equal(binding.dropout(bad, Dropout(0.4, 3), residual=res), binding.dropout(x, Dropout(0.4, 3), residual=res))


def test_gradient_is_the_same_mask():
    """<dy, dropout(x)> is linear in x: its difference along one element is dropout(dy) there."""
    import torch
    x, dy = _rand((9, 40), "fp32", 1), _rand((9, 40), "fp32", 2)
    drop = Dropout(0.5, 77, 1)
    dx = binding.dropout(dy, drop)
    for at in [(0, 0), (3, 17), (8, 39), (5, 8)]:
        hi, lo = x.clone(), x.clone()
        hi[at] += 1
        lo[at] -= 1
        diff = (dy.double() * (binding.dropout(hi, drop).double() - binding.dropout(lo, drop).double())).sum() / 2
        # three roundings of values up to 2 (|x| + 1) on either side, times |dy|
        assert abs(float(diff - dx[at])) <= 8 * 2.0**-24 * 2 * (abs(float(x[at])) + 1) * abs(float(dy[at])) + 1e-30


def test_streams_and_graphs():
    import torch
    x, r = _rand((200, 512), "bf16", 1), _rand((200, 512), "bf16", 2)
    want = binding.dropout(x, Dropout(0.1, 4), residual=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.dropout(x, Dropout(0.1, 4), residual=r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.dropout(x, Dropout(0.1, 4), residual=r, out=out)
    for _ in range(2):
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_argument_checks():
    import torch
    x = _rand((8, 16), "bf16", 1)
    with pytest.raises(TypeError):
        binding.dropout(x.half(), Dropout(0.1))
    for bad in (dict(residual=x.float()), dict(out=x[:4]), dict(residual=x.t()), dict(out=torch.empty(16, 8, dtype=x.dtype, device="cuda").t())):
        with pytest.raises(ValueError):
            binding.dropout(x, Dropout(0.1), **bad)
    with pytest.raises(ValueError):
        binding.dropout(x.cpu(), Dropout(0.1))
    with pytest.raises(binding.CmoeError) as e:
        binding.dropout(x, Dropout(1.0))
    assert e.value.status == -1
    assert binding.dropout(x[:0], Dropout(0.1)).shape == (0, 16) and binding.dropout(x[:, :0], Dropout(0.1)).shape == (8, 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_contiguous_rows_of_any_width(dtype):
    """Widths whose rows start inside a vector of the flat array, at every place of it, in batches that end inside one; the same
    values from a matrix that starts off a 16-byte boundary, and nothing written behind the last element."""
    import torch
    for cols in list(range(9, 42)) + [255, 257, 511, 1001]:
        for rows in (1, 2, 67):
            x, r = _rand((rows, cols), dtype, cols), _rand((rows, cols), dtype, cols + 1)
            drop = Dropout(0.3, 2**40 + cols, 2**35, 11)
            keep = ao.keep_mask(rows, cols, 0.3, drop.seed, drop.offset, 11)
            room = torch.full((rows * cols + 16,), 7.0, dtype=x.dtype, device="cuda")
            got = binding.dropout(x, drop, out=room[:rows * cols].view(rows, cols))
            np.testing.assert_array_equal(_host(got) != 0, keep & (_host(x) != 0))
            assert (room[rows * cols:] == 7).all()
            both = binding.dropout(x, drop, residual=r)
            _check(both, ao.dropout(_host(x), 0.3, drop.seed, drop.offset, 11, _host(r)), np.abs(_host(x)) * 1.43 + np.abs(_host(r)), dtype)
            off = torch.empty(rows * cols + 1, dtype=x.dtype, device="cuda")[1:].view(rows, cols).copy_(x)
            assert torch.equal(binding.dropout(off, drop, residual=r), both)
