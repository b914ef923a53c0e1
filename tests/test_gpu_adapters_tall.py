"""-m gpu: adapters of higher ranks on batches long enough for tiles of 128 rows (tcgen05), against the 64-bit oracle.

Tolerances as for the other adapters: sums over k products are chains of at most (k / 8 + 64) steps, here one MMA for 16 products and
the sums of up to eight blocks; bf16 results keep 15 bits of the narrow middle; one rounding at the end."""
import numpy as np
import pytest

from oracle import adapters_oracle as ao
from paper_2502_04416_b200 import binding, workloads as wl
from paper_2502_04416_b200.binding import Dropout
from tests import parity
from tests.test_gpu_adapters import check_backward, check_forward, make

pytestmark = pytest.mark.gpu

SHAPES = [  # rows, adapters, rank, d_in, d_out, order of the rows
    (1024, 1, 64, 72, 136, None),          # one adapter, tiles full
    (1025, 1, 40, 136, 64, None),          # one row in the last tile
    (1030, 32, 48, 264, 96, "mixed"),      # an adapter's tile is a quarter full; rows without one
    (1151, 7, 56, 200, 1000, "mixed"),     # widths that end inside a block
    (1300, 40, 64, 8, 8, "mixed"),         # the narrowest
    (1500, 3, 64, 520, 24, "skewed"),
    (2100, 5, 48, 1376, 40, "sorted"),     # d_in spread over a cluster, one block of d_out
    (2100, 5, 48, 40, 1376, "sorted"),     # and the other way
    (2048, 2, 64, 64, 64, "none"),
    (4096, 3, 32, 104, 8, "mixed"),        # ranks up to 32: the other kernel for the weights' gradients
    (4100, 1, 24, 8, 264, None),
    (5000, 60, 32, 64, 72, "mixed")]


@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape):
    s = make("bf16", *shape[:5], ids=shape[5], dy=True)
    out, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=s["base"], want_z=True)
    check_forward(s, "bf16", out, z)
    got = binding.adapter_backward(s["dy"], s["x"], z, s["a"], s["b"], s["ids"], s["scale"], dx_base=s["dx_base"])
    check_backward(s, "bf16", got, z)
    assert binding.adapter_status() == 0


@pytest.mark.parametrize("ids", [None, "mixed"])
@pytest.mark.parametrize("rows,r,drop", [(1100, 64, Dropout(0.1, 2**40 + 1, 3, 5)), (4097, 24, Dropout(0.5, 7, 2**40))])
def test_dropout_parts_and_repeats(rows, r, drop, ids):
    import torch
    s = make("bf16", rows, 5 if ids else 1, r, 200, 136, ids=ids, seed=r, dy=True)
    args = (s["a"], s["b"], s["ids"], s["scale"])
    out, z = binding.adapter_forward(s["x"], *args, dropout=drop, want_z=True)
    check_forward(s, "bf16", out, z, drop, base=False)
    got = binding.adapter_backward(s["dy"], s["x"], z, *args, dropout=drop)
    check_backward(s, "bf16", got, z, drop, dx_base=False)
    again = binding.adapter_backward(s["dy"], s["x"], z, *args, dropout=drop)
    assert all(torch.equal(u, v) for u, v in zip(got, again))
    only_dx = binding.adapter_backward(s["dy"], None, None, *args, dropout=drop, want_grads=False)[0]
    _, ga, gb = binding.adapter_backward(s["dy"], s["x"], z, *args, dropout=drop, want_dx=False)
    assert torch.equal(only_dx, got[0]) and torch.equal(ga, got[1]) and torch.equal(gb, got[2])
    # a dropped input may hold anything
    keep = torch.from_numpy(ao.keep_mask(rows, 200, drop.p, drop.seed, drop.offset, drop.row0)).cuda()
    bad = torch.where(keep, s["x"], torch.full_like(s["x"], float("nan")))
    for u, v in zip(binding.adapter_forward(bad, *args, dropout=drop, want_z=True), (out, z)):
        assert torch.equal(u, v)
    bad_g = binding.adapter_backward(s["dy"], bad, z, *args, dropout=drop)
    assert all(torch.equal(u, v) for u, v in zip(bad_g, got))


@pytest.mark.parametrize("rows,r", [(1200, 48), (4200, 24)])
def test_rows_and_adapters_do_not_see_each_other(rows, r):
    """NaN, infinities and the type's lowest value in some rows, and in one adapter's weights, change no bit of the other rows and the
    other adapters' gradients; a permutation of the batch permutes the results."""
    import torch
    n = 6
    s = make("bf16", rows, n, r, 136, 200, seed=5, dy=True)
    args = (s["a"], s["b"], s["ids"], s["scale"])
    want, z = binding.adapter_forward(s["x"], *args, base=s["base"], want_z=True)
    grads = binding.adapter_backward(s["dy"], s["x"], z, *args, dx_base=s["dx_base"])
    bad = s["x"].clone()
    hit = torch.arange(rows, device="cuda") % 3 == 1
    for i, v in enumerate((float("nan"), float("inf"), torch.finfo(bad.dtype).min)):
        bad[torch.nonzero(hit).flatten()[i::3]] = v
    got, bad_z = binding.adapter_forward(bad, *args, base=s["base"], want_z=True)
    assert torch.equal(got[~hit], want[~hit]) and torch.equal(bad_z[~hit], z[~hit])
    a, b, own = s["a"].clone(), s["b"].clone(), s["ids"] == 2
    a[2], b[2] = float("nan"), float("inf")
    got = binding.adapter_forward(s["x"], a, b, *args[2:], base=s["base"])
    assert torch.equal(got[~own], want[~own])
    bad_dy, bad_x = s["dy"].clone(), s["x"].clone()
    bad_dy[own], bad_x[own] = float("nan"), float("inf")
    dx, ga, gb = binding.adapter_backward(bad_dy, bad_x, z, a, b, *args[2:], dx_base=s["dx_base"])
    rest = torch.arange(n, device="cuda") != 2
    assert torch.equal(dx[~own], grads[0][~own]) and torch.equal(ga[rest], grads[1][rest]) and torch.equal(gb[rest], grads[2][rest])
    order = torch.randperm(rows, generator=torch.Generator().manual_seed(0)).cuda()
    got = binding.adapter_forward(s["x"][order], s["a"], s["b"], s["ids"][order], s["scale"], base=s["base"][order])
    assert torch.equal(got, want[order])


def test_views_in_place_and_rows_behind_the_batch():
    import torch
    rows, n, r, d_in, d_out = 1100, 4, 40, 104, 72
    s = make("bf16", rows, n, r, d_in, d_out, seed=3, dy=True)
    args = (s["a"], s["b"], s["ids"], s["scale"])
    want, z = binding.adapter_forward(s["x"], *args, base=s["base"], want_z=True)
    grads = binding.adapter_backward(s["dy"], s["x"], z, *args, dx_base=s["dx_base"])
    wide = torch.full((rows + 2, 8 + d_in + 8 + d_out + 8 + d_out + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    at = [8, 16 + d_in, 24 + d_in + d_out]
    xs, bs, os_ = wide[1:-1, at[0]:at[0] + d_in], wide[1:-1, at[1]:at[1] + d_out], wide[1:-1, at[2]:at[2] + d_out]
    xs.copy_(s["x"]); bs.copy_(s["base"])
    before = wide.clone()
    binding.adapter_forward(xs, *args, base=bs, out=os_)
    assert torch.equal(os_, want)
    os_.copy_(before[1:-1, at[2]:at[2] + d_out])
    assert torch.equal(wide, before)
    got = binding.adapter_backward(s["dy"], xs, z, *args, dx_base=s["dx_base"])
    assert all(torch.equal(u, v) for u, v in zip(got, grads))
    own, own_dx = s["base"].clone(), s["dx_base"].clone()
    binding.adapter_forward(s["x"], *args, base=own, out=own)
    binding.adapter_backward(s["dy"], s["x"], z, *args, dx_base=own_dx, dx=own_dx)
    assert torch.equal(own, want) and torch.equal(own_dx, grads[0])
    # a batch of the first 1030 rows of longer matrices
    k = 1030
    out, zz, dx = s["base"].clone(), torch.full((rows, r), 9.0, device="cuda"), s["dx_base"].clone()
    ids = s["ids"][:k].contiguous()
    binding.adapter_forward(s["x"][:k], s["a"], s["b"], ids, s["scale"], base=s["base"][:k], out=out[:k], z=zz[:k])
    binding.adapter_backward(s["dy"][:k], s["x"][:k], zz[:k].contiguous(), s["a"], s["b"], ids, s["scale"], dx=dx[:k])
    assert torch.equal(out[k:], s["base"][k:]) and (zz[k:] == 9).all() and torch.equal(dx[k:], s["dx_base"][k:])


@pytest.mark.parametrize("rows,r", [(1200, 56), (4200, 32)])
def test_streams_graphs_and_scratch(rows, r):
    import torch
    s = make("bf16", rows, 5, r, 256, 320, seed=4, dy=True)
    args = (s["a"], s["b"], s["ids"], s["scale"])
    want, z = binding.adapter_forward(s["x"], *args, base=s["base"], want_z=True)
    grads = binding.adapter_backward(s["dy"], s["x"], z, *args)
    sides = [torch.cuda.Stream() for _ in range(3)]
    got = []
    torch.cuda.synchronize()
    for st in sides * 2:                                                                  # calls that run side by side
        got.append((binding.adapter_forward(s["x"], *args, base=s["base"], stream=st),
                    *binding.adapter_backward(s["dy"], s["x"], z, *args, stream=st)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(u, v) for u, v in zip(g, (want, *grads)))
    need = [binding.adapter_scratch_bytes(5, r, 256, 320, torch.bfloat16, rows, backward=k) for k in (False, True)]
    scr = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in need]         # contents do not matter
    out, dx, ga, gb = (torch.empty_like(t) for t in (want, *grads))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.adapter_forward(s["x"], *args, base=s["base"], out=out, z=z, scratch=scr[0])
        binding.adapter_backward(s["dy"], s["x"], z, *args, dx=dx, grad_a=ga, grad_b=gb, scratch=scr[1])
    for ids in (s["ids"].clone(), s["ids"].flip(0).contiguous(), torch.full_like(s["ids"], -1), torch.zeros_like(s["ids"])):
        s["ids"].copy_(ids)                                                               # the captured calls read the ids anew
        for t in (out, dx, ga, gb, z):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        w, wz = binding.adapter_forward(s["x"], *args, base=s["base"], want_z=True)
        assert torch.equal(out, w) and torch.equal(z, wz)
        assert all(torch.equal(u, v) for u, v in zip((dx, ga, gb), binding.adapter_backward(s["dy"], s["x"], wz, *args)))


def test_long_batch():
    """Offsets past 32 bits in bytes (x of 2.2 GB, out of 4.4), rows of two adapters in turn: some rows against the oracle, and the
    gradients against sums that torch forms in 64 bits."""
    import torch
    rows, d_in, d_out, r = 270_000, 4096, 8192, 40
    g = torch.Generator("cuda").manual_seed(0)
    x = torch.empty(rows, d_in, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    a = (torch.randn(2, r, d_in, generator=g, device="cuda") / 64).bfloat16()
    b = torch.randn(2, d_out, r, generator=g, device="cuda").bfloat16()
    ids = (torch.arange(rows, device="cuda") % 2).to(torch.int32)
    out, z = binding.adapter_forward(x, a, b, ids, None, want_z=True)
    for lo in (0, rows // 2, rows - 40):
        s = dict(x=x[lo:lo + 40], a=a, b=b, scale=torch.ones(2), ids_np=np.arange(lo, lo + 40) % 2)
        check_forward(s, "bf16", out[lo:lo + 40], z[lo:lo + 40], base=False)
    dx, ga, gb = binding.adapter_backward(out, x, z, a, b, ids, None)
    for lo in (0, rows - 40):
        s = dict(x=x[lo:lo + 40], a=a, b=b, scale=torch.ones(2), ids_np=np.arange(lo, lo + 40) % 2, dy=out[lo:lo + 40])
        check_backward(s, "bf16", (dx[lo:lo + 40], None, None), z[lo:lo + 40], dx_base=False)
    for i in (0, 1):
        cols = torch.tensor([0, 7, 4095, 2048], device="cuda")
        for got, v, zz in ((gb[i][cols], out[i::2][:, cols], z[i::2]),):
            want = v.double().t() @ zz.double()
            mag = v.double().abs().t() @ zz.double().abs()
            bound = 2.0**-9 * want.abs() + 1.01 * ((2 * rows / 8 + 64) * 2.0**-23 + 2.0**-15 + 2.0**-21) * mag
            assert ((got.double() - want).abs() <= bound).all()
        e = out[i::2].double() @ b[i].double()
        want, mag = e.t() @ x[i::2][:, cols].double(), e.abs().t() @ x[i::2][:, cols].double().abs()
        e_mag = (out[i::2].double().abs() @ b[i].double().abs()).t() @ x[i::2][:, cols].double().abs()
        bound = 2.0**-9 * want.abs() + 1.01 * (((2 * rows / 8 + 64) * 2.0**-23 + 2.0**-15 + 2.0**-21) * mag + (d_out / 8 + 64) * 2.0**-23 * e_mag)
        assert ((ga[i][:, cols].double() - want).abs() <= bound).all()
        del e


@pytest.mark.parametrize("mixed", [True, False])
def test_beside_a_layer(mixed):
    import torch
    rows = 1100
    inp = wl.make_inputs(wl.Workload("adapted", wl.LayerShape(256, 1024, 8, 2, 2, "bf16"), (rows,), seed=3))
    layer = parity.gpu_layer(inp.layers[0], rows)
    x = parity.to_device(inp.x, "bf16")
    s = make("bf16", rows, 5, 40, 256, 256, ids="mixed" if mixed else None, seed=1)
    plain = layer.forward(x)
    want = binding.adapter_forward(x, s["a"], s["b"], s["ids"], s["scale"], base=plain)
    for _ in range(2):
        assert torch.equal(layer.forward_adapted(x, s["a"], s["b"], s["ids"], s["scale"]), want)
    s["x"], s["base"] = x, plain
    check_forward(s, "bf16", want, None)
    layer.destroy()
