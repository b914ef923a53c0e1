"""-m gpu: low-rank adapters of many requests (cmoe_adapter_forward / _backward, cmoe_ffn_forward_adapted) against the 64-bit oracle.

Tolerances count roundings.  A sum of k products held in 32 bits is off by at most k * 2^-23 of the sum of magnitudes (MMA sums cut
off rather than round, a whole step of 2^-23 each); chains are at most (length / 8 + 64) long: two MMAs for 32 products, then the
sums of warps and blocks.  On fp32 operands a chain has one rounding a product.  bf16 results keep 15 bits of the narrow middle, which
is 2^-15 of its magnitude.  The result is rounded once to its type: eps / 2."""
import numpy as np
import pytest

from oracle import adapters_oracle as ao, cmoe_oracle as oracle
from paper_2502_04416_b200 import binding, workloads as wl
from paper_2502_04416_b200.binding import Dropout
from tests import parity

pytestmark = pytest.mark.gpu

DT = {"bf16": "bfloat16", "fp32": "float32"}


def _eps(dtype):
    import torch
    return torch.finfo(getattr(torch, DT[dtype])).eps


def _host(t):
    return t.double().cpu().numpy()


def _chain(length, dtype):
    return (length / 8 + 64 if dtype == "bf16" else length + 64) * 2.0**-23


def make(dtype, rows, n, r, d_in, d_out, ids="mixed", seed=0, dy=False):
    """Rows, adapters and scales; ids: the adapter of each row ("mixed": -1 and n among them)."""
    import torch
    g = torch.Generator("cuda").manual_seed(1000 * seed + rows + r)
    dt = getattr(torch, DT[dtype])

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)

    s = dict(x=normal(rows, d_in), a=normal(n, r, d_in, std=d_in**-0.5), b=normal(n, d_out, r, std=r**-0.5), base=normal(rows, d_out),
             scale=torch.rand(n, generator=g, device="cuda") * 3 + 0.25)
    rng = np.random.default_rng(seed + rows)
    if ids == "mixed":
        ids = rng.integers(-1, n + 1, rows)
    elif ids == "sorted":
        ids = np.sort(rng.integers(0, n, rows))
    elif ids == "skewed":                        # one adapter has nearly all rows, many have none
        ids = np.where(rng.random(rows) < 0.9, n // 2, rng.integers(0, n, rows))
    elif ids == "none":
        ids = np.full(rows, -1)
    s["ids_np"] = np.zeros(rows, dtype=np.int64) if ids is None else np.asarray(ids)
    s["ids"] = None if ids is None else torch.from_numpy(np.asarray(ids).astype(np.int32)).cuda()
    if dy:
        s["dy"] = normal(rows, d_out)
        s["dx_base"] = normal(rows, d_in)
    return s


def _mask(rows, cols, drop):
    if drop is None:
        return np.ones((rows, cols))
    return ao.keep_mask(rows, cols, drop.p, drop.seed, drop.offset, drop.row0) * (65536 / (65536 - ao.threshold(drop.p)))


def check_forward(s, dtype, got, z, drop=None, base=True):
    x, a, b, sc = _host(s["x"]), _host(s["a"]), _host(s["b"]), _host(s["scale"])
    xd = x * _mask(*x.shape, drop)
    base = _host(s["base"]) if base else None
    want, zw = ao.adapter_forward(xd, a, b, s["ids_np"], sc, base)
    mag, zmag = ao.adapter_forward(np.abs(xd), np.abs(a), np.abs(b), s["ids_np"], sc, None)
    rel = _chain(x.shape[1], dtype) + _chain(a.shape[1], dtype) + (2.0**-15 if dtype == "bf16" else 0)
    bound = _eps(dtype) / 2 * np.abs(want) + (1 + _eps(dtype)) * (rel * mag + 2.0**-23 * (np.abs(want) + mag))
    err = np.abs(_host(got) - want)
    assert np.isfinite(err).all() and (err <= bound).all(), (err - bound).max()
    if z is not None:
        err = np.abs(_host(z) - zw)
        assert (err <= (_chain(x.shape[1], dtype) + 2.0**-22) * zmag).all()
    none = (s["ids_np"] < 0) | (s["ids_np"] >= a.shape[0])
    if base is not None:
        np.testing.assert_array_equal(_host(got)[none], base[none])     # rows without an adapter keep the projection's bits


SHAPES = [  # rows, adapters, rank, d_in, d_out
    (1, 1, 8, 8, 8), (1, 8, 8, 4096, 4096), (2, 3, 16, 40, 24), (15, 1, 8, 256, 1024), (16, 2, 24, 72, 264), (17, 5, 32, 256, 96),
    (64, 64, 16, 512, 520), (65, 1, 64, 264, 128), (200, 24, 32, 1000, 648), (255, 300, 8, 128, 64), (256, 1024, 40, 96, 136),
    (257, 3, 16, 256, 256), (300, 1024, 8, 64, 72), (513, 2, 48, 1376, 40), (1000, 7, 56, 248, 376), (1030, 3, 64, 520, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dtype, shape):
    s = make(dtype, *shape)
    out, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=s["base"], want_z=True)
    check_forward(s, dtype, out, z)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ids", [None, "sorted", "skewed", "none"])
@pytest.mark.parametrize("rows", [100, 700])
def test_forward_orders_and_dropout(dtype, ids, rows):
    for r, drop in ((8, Dropout(0.1, 2**40 + 1, 3, 5)), (16, None), (32, Dropout(0.5, 7)), (64, Dropout(0.05, 8, 2**40))):
        s = make(dtype, rows, 6, r, 136, 200, ids=ids, seed=r)
        out, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=s["base"], dropout=drop, want_z=True)
        check_forward(s, dtype, out, z, drop)
        out = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], dropout=drop)
        check_forward(s, dtype, out, None, drop, base=False)


def _plain_scale(s):
    import torch
    s["scale"] = torch.ones_like(s["scale"])
    return s


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [40, 400])
def test_forward_views_in_place_and_without_scale(dtype, rows):
    import torch
    n, r, d_in, d_out = 4, 16, 104, 72
    s = _plain_scale(make(dtype, rows, n, r, d_in, d_out, seed=3))
    want = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=s["base"])
    assert torch.equal(binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], None, base=s["base"]), want)
    own = s["base"].clone()
    binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=own, out=own)
    assert torch.equal(own, want)
    # x, base and out as column slices of one wide matrix, with rows before and after
    wide = torch.full((rows + 2, 8 + d_in + 8 + d_out + 8 + d_out + 16), 7.0, dtype=s["x"].dtype, device="cuda")
    at = [8, 16 + d_in, 24 + d_in + d_out]
    xs, bs, os_ = wide[1:-1, at[0]:at[0] + d_in], wide[1:-1, at[1]:at[1] + d_out], wide[1:-1, at[2]:at[2] + d_out]
    xs.copy_(s["x"]); bs.copy_(s["base"])
    before = wide.clone()
    binding.adapter_forward(xs, s["a"], s["b"], s["ids"], s["scale"], base=bs, out=os_)
    assert torch.equal(os_, want)
    os_.copy_(before[1:-1, at[2]:at[2] + d_out])
    assert torch.equal(wide, before)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_row_does_not_see_the_others(dtype):
    """Rows of NaN, infinities and the type's lowest value beside a row, in the same tile or not, change no bit of it; a
    permutation of the batch permutes the results."""
    import torch
    s = make(dtype, 90, 3, 16, 128, 96, seed=5)
    want = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], base=s["base"])
    bad = s["x"].clone()
    hit = torch.arange(90, device="cuda") % 3 == 1
    for i, v in enumerate((float("nan"), float("inf"), torch.finfo(bad.dtype).min)):
        bad[torch.nonzero(hit).flatten()[i::3]] = v
    got = binding.adapter_forward(bad, s["a"], s["b"], s["ids"], s["scale"], base=s["base"])
    assert torch.equal(got[~hit], want[~hit])
    order = torch.randperm(90, generator=torch.Generator().manual_seed(0)).cuda()
    got = binding.adapter_forward(s["x"][order], s["a"], s["b"], s["ids"][order], s["scale"], base=s["base"][order])
    assert torch.equal(got, want[order])


def test_dropped_inputs_may_hold_anything():
    import torch
    for dtype in ("bf16", "fp32"):
        s = make(dtype, 50, 2, 8, 64, 64, seed=6)
        drop = Dropout(0.3, 21)
        keep = torch.from_numpy(ao.keep_mask(50, 64, drop.p, drop.seed)).cuda()
        bad = torch.where(keep, s["x"], torch.full_like(s["x"], float("nan")))
        args = (s["a"], s["b"], s["ids"], s["scale"])
        for u, v in zip(binding.adapter_forward(bad, *args, dropout=drop, want_z=True),
                        binding.adapter_forward(s["x"], *args, dropout=drop, want_z=True)):
            assert torch.equal(u, v)


def check_backward(s, dtype, got, z, drop=None, dx_base=True):
    x, a, b, sc, dy, zz = (_host(t) for t in (s["x"], s["a"], s["b"], s["scale"], s["dy"], z))
    mask = _mask(*x.shape, drop)
    base = _host(s["dx_base"]) if dx_base else None
    want = ao.adapter_backward(dy, x * mask, zz, a, b, s["ids_np"], sc, mask, base)
    mag = ao.adapter_backward(np.abs(dy), np.abs(x) * mask, np.abs(zz), np.abs(a), np.abs(b), s["ids_np"], sc, mask, None)
    cut = 2.0**-15 if dtype == "bf16" else 0
    rows = len(x)
    rel = [_chain(dy.shape[1], dtype) + _chain(a.shape[1], dtype) + cut, _chain(dy.shape[1], dtype) + _chain(2 * rows, dtype) + cut,
           _chain(2 * rows, dtype) + cut]
    for i, name in enumerate(("dx", "grad_a", "grad_b")):
        if got[i] is None:
            continue
        bound = _eps(dtype) / 2 * np.abs(want[i]) + (1 + _eps(dtype)) * ((rel[i] + 2.0**-21) * mag[i] + 2.0**-23 * np.abs(want[i]))
        err = np.abs(_host(got[i]) - want[i])
        assert np.isfinite(err).all() and (err <= bound).all(), (name, (err - bound).max())
    if got[1] is not None:
        for k in set(range(a.shape[0])) - set(s["ids_np"].tolist()):
            assert not got[1][k].any() and not got[2][k].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dtype, shape):
    s = make(dtype, *shape, dy=True)
    _, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], want_z=True)
    got = binding.adapter_backward(s["dy"], s["x"], z, s["a"], s["b"], s["ids"], s["scale"], dx_base=s["dx_base"])
    check_backward(s, dtype, got, z)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ids", [None, "sorted", "skewed", "none"])
def test_backward_orders_dropout_and_parts(dtype, ids):
    import torch
    for r, rows, drop in ((8, 700, Dropout(0.1, 2**40 + 1, 3, 5)), (16, 90, None), (32, 333, Dropout(0.5, 7)), (64, 260, Dropout(0.05, 8, 2**40))):
        s = make(dtype, rows, 6, r, 136, 200, ids=ids, seed=r, dy=True)
        _, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], dropout=drop, want_z=True)
        args = (s["dy"], s["x"], z, s["a"], s["b"], s["ids"], s["scale"])
        got = binding.adapter_backward(*args, dropout=drop)
        check_backward(s, dtype, got, z, drop, dx_base=False)
        again = binding.adapter_backward(*args, dropout=drop)
        assert all(torch.equal(u, v) for u, v in zip(got, again))       # sums over rows have a fixed order
        only_dx = binding.adapter_backward(s["dy"], None, None, *args[3:], dropout=drop, want_grads=False)
        assert torch.equal(only_dx[0], got[0]) and only_dx[1] is None and only_dx[2] is None
        only_w = binding.adapter_backward(*args, dropout=drop, want_dx=False)
        assert only_w[0] is None and torch.equal(only_w[1], got[1]) and torch.equal(only_w[2], got[2])
        own = s["dx_base"].clone()
        binding.adapter_backward(*args, dropout=drop, dx_base=own, dx=own)
        check_backward(s, dtype, (own, None, None), z, drop)


def test_backward_of_no_rows_zeroes_the_gradients():
    import torch
    s = make("bf16", 4, 3, 8, 64, 32, dy=True)
    z = torch.zeros(0, 8, device="cuda")
    ga, gb = torch.full_like(s["a"], 5.0), torch.full_like(s["b"], 5.0)
    dx, _, _ = binding.adapter_backward(s["dy"][:0], s["x"][:0], z, s["a"], s["b"], s["ids"][:0], s["scale"], grad_a=ga, grad_b=gb)
    assert dx.shape == (0, 64) and not ga.any() and not gb.any()
    assert binding.adapter_forward(s["x"][:0], s["a"], s["b"], s["ids"][:0], s["scale"]).shape == (0, 32)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gradients_against_differences(dtype):
    """The loss <dy, out> is linear in x, A and B one at a time, so a difference of one element has no truncation error; only the
    forward's roundings of that element's contribution remain."""
    import torch
    s = make(dtype, 70, 2, 8, 64, 48, seed=9, dy=True)
    drop = Dropout(0.2, 31)

    def second(z, b, scale):                                             # the second product in 64 bits, from the kernel's z
        out = np.zeros((70, 48))
        for t, k in enumerate(s["ids_np"]):
            if 0 <= k < 2:
                out[t] = scale[k] * (b[k] @ z[t])
        return out

    def loss(**kw):
        """The loss, and how far 32-bit sums of z may put it off."""
        t = {**s, **kw}
        _, z = binding.adapter_forward(t["x"], t["a"], t["b"], t["ids"], t["scale"], dropout=drop, want_z=True)
        x, a, b, sc = (_host(t[k]) for k in ("x", "a", "b", "scale"))
        mag, _ = ao.adapter_forward(np.abs(x) * _mask(70, 64, drop), np.abs(a), np.abs(b), s["ids_np"], sc)
        return float((_host(s["dy"]) * second(_host(z), b, sc)).sum()), float((np.abs(_host(s["dy"])) * mag).sum()) * (_chain(64, dtype) + 2.0**-22)

    _, z = binding.adapter_forward(s["x"], s["a"], s["b"], s["ids"], s["scale"], dropout=drop, want_z=True)
    grads = binding.adapter_backward(s["dy"], s["x"], z, s["a"], s["b"], s["ids"], s["scale"], dropout=drop)
    mask = _mask(70, 64, drop)
    mags = ao.adapter_backward(*(np.abs(_host(t)) for t in (s["dy"], s["x"])), np.abs(_host(z)), *(np.abs(_host(s[k])) for k in "ab"),
                               s["ids_np"], _host(s["scale"]), mask)
    mags = (mags[0], mags[1] * mask.max(), mags[2])
    inner = _chain(48, dtype) + _chain(140, dtype) + 2.0**-21 + (2.0**-15 if dtype == "bf16" else 0)
    rng = np.random.default_rng(2)
    for name, grad, mag in zip(("x", "a", "b"), grads, mags):
        for _ in range(6):
            at = tuple(int(rng.integers(0, n)) for n in grad.shape)
            hi, lo = s[name].clone(), s[name].clone()
            hi[at], lo[at] = 4.0, -4.0                                   # exact in both types: the step is 8
            (up, off_up), (down, off_down) = loss(**{name: hi}), loss(**{name: lo})
            allowed = _eps(dtype) * abs(float(grad[at])) + 1.01 * inner * mag[at] + (off_up + off_down) / 8
            assert abs((up - down) / 8 - float(grad[at])) <= allowed


def test_many_rows_of_one_long_batch():
    """Enough rows that offsets pass 32 bits in bytes (x of 2.2 GB, out of 4.4): the last rows against the oracle."""
    import torch
    rows, d_in, d_out, r = 270_000, 4096, 8192, 8
    g = torch.Generator("cuda").manual_seed(0)
    x = torch.empty(rows, d_in, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    a = (torch.randn(2, r, d_in, generator=g, device="cuda") / 64).bfloat16()
    b = torch.randn(2, d_out, r, generator=g, device="cuda").bfloat16()
    ids = (torch.arange(rows, device="cuda") % 2).to(torch.int32)
    out, z = binding.adapter_forward(x, a, b, ids, None, want_z=True)
    for lo in (0, rows // 2, rows - 40):
        s = dict(x=x[lo:lo + 40], a=a, b=b, scale=torch.ones(2), ids_np=np.arange(lo, lo + 40) % 2)
        check_forward(s, "bf16", out[lo:lo + 40], z[lo:lo + 40], base=False)


def test_streams_graphs_and_scratch():
    import torch
    for rows in (60, 600):
        s = make("bf16", rows, 5, 16, 256, 320, seed=4, dy=True)
        args = (s["a"], s["b"], s["ids"], s["scale"])
        want, z = binding.adapter_forward(s["x"], *args, base=s["base"], want_z=True)
        grads = binding.adapter_backward(s["dy"], s["x"], z, *args)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = binding.adapter_forward(s["x"], *args, base=s["base"], stream=side)
        got_g = binding.adapter_backward(s["dy"], s["x"], z, *args, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want) and all(torch.equal(u, v) for u, v in zip(got_g, grads))
        need = [max(binding.adapter_scratch_bytes(5, 16, 256, 320, torch.bfloat16, rows, backward=k), 1) for k in (False, True)]
        scr = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in need]      # contents do not matter
        out, dx, ga, gb = (torch.empty_like(t) for t in (want, *grads))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.adapter_forward(s["x"], *args, base=s["base"], out=out, z=z, scratch=scr[0])
            binding.adapter_backward(s["dy"], s["x"], z, *args, dx=dx, grad_a=ga, grad_b=gb, scratch=scr[1])
        for _ in range(3):
            for t in (out, dx, ga, gb, z):
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and all(torch.equal(u, v) for u, v in zip((dx, ga, gb), grads))
        ids2 = s["ids"].flip(0).contiguous()                                              # the captured call reads the ids anew
        want2 = binding.adapter_forward(s["x"], s["a"], s["b"], ids2, s["scale"], base=s["base"])
        s["ids"].copy_(ids2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want2)


def test_rows_behind_the_batch_are_left_alone():
    import torch
    for rows in (37, 300):
        s = make("bf16", rows + 20, 3, 8, 64, 64, seed=8, dy=True)
        out, z = s["base"].clone(), torch.full((rows + 20, 8), 9.0, device="cuda")
        dx = s["dx_base"].clone()
        ids = s["ids"][:rows].contiguous()
        binding.adapter_forward(s["x"][:rows], s["a"], s["b"], ids, s["scale"], base=s["base"][:rows], out=out[:rows], z=z[:rows])
        binding.adapter_backward(s["dy"][:rows], s["x"][:rows], z[:rows].contiguous(), s["a"], s["b"], ids, s["scale"], dx=dx[:rows])
        assert torch.equal(out[rows:], s["base"][rows:]) and (z[rows:] == 9).all() and torch.equal(dx[rows:], s["dx_base"][rows:])


def test_refused_launches_are_reported_once():
    """A launch into a broken capture fails with CMOE_ERR_CUDA and leaves nothing behind for the next call."""
    import torch
    from cuda.bindings import runtime as rt
    s = make("bf16", 300, 3, 8, 64, 64)
    args = (s["x"], s["a"], s["b"], s["ids"], s["scale"])
    want = binding.adapter_forward(*args)
    out = torch.empty_like(want)
    scr = torch.empty(binding.adapter_scratch_bytes(3, 8, 64, 64, torch.bfloat16, 300), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert rt.cudaStreamBeginCapture(side.cuda_stream, rt.cudaStreamCaptureMode.cudaStreamCaptureModeRelaxed)[0] == rt.cudaError_t.cudaSuccess
    assert rt.cudaStreamSynchronize(side.cuda_stream)[0] != rt.cudaError_t.cudaSuccess
    with pytest.raises(binding.CmoeError) as e:
        binding.adapter_forward(*args, out=out, scratch=scr, stream=side)
    assert e.value.status == -5
    rt.cudaStreamEndCapture(side.cuda_stream)
    rt.cudaGetLastError()
    assert torch.equal(binding.adapter_forward(*args), want)


def test_argument_checks():
    import torch
    s = make("bf16", 20, 3, 8, 64, 32, dy=True)
    ok = dict(row_adapter=s["ids"], scale=s["scale"])
    for bad in (dict(row_adapter=s["ids"].long()), dict(row_adapter=s["ids"][:5]), dict(scale=s["scale"].double()), dict(scale=s["scale"][:2]),
                dict(base=s["base"].float()), dict(base=s["base"][:, :16]), dict(out=s["base"][:3]), dict(z=torch.zeros(20, 16, device="cuda")),
                dict(scratch=torch.zeros(8, device="cuda"))):
        with pytest.raises(ValueError):
            binding.adapter_forward(s["x"], s["a"], s["b"], **{**ok, **bad})
    for x, a, b in ((s["x"][:, :56], s["a"], s["b"]), (s["x"].float(), s["a"], s["b"]), (s["x"], s["a"][:2], s["b"]),
                    (s["x"], s["a"].transpose(1, 2), s["b"]), (s["x"].cpu(), s["a"], s["b"])):
        with pytest.raises(ValueError):
            binding.adapter_forward(x, a, b, **ok)
    z = torch.zeros(20, 8, device="cuda")
    for bad in (dict(z=z[:4]), dict(dx_base=s["x"].float()), dict(grad_a=s["b"]), dict(grad_a=s["a"].clone(), grad_b=s["b"].float())):
        with pytest.raises(ValueError):
            binding.adapter_backward(s["dy"], s["x"], **{**dict(z=z, a=s["a"], b=s["b"]), **ok, **bad})
    with pytest.raises(binding.CmoeError) as e:
        binding.adapter_forward(s["x"], s["a"][:, :4].contiguous(), s["b"][..., :4].contiguous(), **ok)      # rank 4
    assert e.value.status == -1
    with pytest.raises(binding.CmoeError) as e:
        binding.adapter_forward(s["x"], s["a"], s["b"], out=s["x"][:, :32])                                # overlaps x
    assert e.value.status == -1


# ------------------------------------------------------------------ beside a layer
@pytest.mark.parametrize("dtype,rows", [("fp32", 64), ("bf16", 1), ("bf16", 16), ("bf16", 300)])
def test_layer_with_an_adapter_per_request(dtype, rows):
    import torch
    w = wl.Workload("adapted", wl.LayerShape(256, 1024, 8, 2, 2, dtype), (rows,), seed=3)
    inp = wl.make_inputs(w)
    layer = parity.gpu_layer(inp.layers[0], rows)
    x = parity.to_device(inp.x, dtype)
    s = make(dtype, rows, 5, 8, 256, 256, seed=1)
    plain = layer.forward(x)
    launches = layer.launch_count()
    want = binding.adapter_forward(x, s["a"], s["b"], s["ids"], s["scale"], base=plain)
    for _ in range(2):
        got = layer.forward_adapted(x, s["a"], s["b"], s["ids"], s["scale"])
        assert torch.equal(got, want)
    assert layer.launch_count() == launches + (2 if rows > 256 else 1)
    s["x"], s["base"] = x, plain
    check_forward(s, dtype, got, None)                                   # the layer's own output is held to the oracle elsewhere
    assert layer.forward_adapted(x[:0], s["a"], s["b"], s["ids"][:0], s["scale"]).shape == (0, 256)
    out = torch.full_like(x, 3.0)
    for bad in (dict(a=s["a"][:, :, :128].contiguous()), dict(b=s["b"][:, :128].contiguous())):
        with pytest.raises((binding.CmoeError, ValueError)):
            layer.forward_adapted(x, **{**dict(a=s["a"], b=s["b"]), **bad}, row_adapter=s["ids"], out=out)
    torch.cuda.synchronize()
    assert (out == 3).all()                                              # refused before anything was launched
    layer.destroy()


def test_layer_hierarchical_with_adapters():
    import torch
    w = wl.shrunk(wl.WORKLOADS["c4_hier_8x7b"], d_model=256, tokens=(40,), m=64, n_outer=3)
    inp = wl.make_inputs(w)
    from paper_2502_04416_b200 import torch_io
    layer = torch_io.layer_from_workload(inp, 40)
    x = parity.to_device(inp.x, "bf16")
    s = make("bf16", 40, 2, 16, 256, 256, seed=2)
    want = binding.adapter_forward(x, s["a"], s["b"], s["ids"], s["scale"], base=layer.forward(x))
    assert torch.equal(layer.forward_adapted(x, s["a"], s["b"], s["ids"], s["scale"]), want)
    layer.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_tuning_step_of_a_sublayer(dtype):
    """All of them together: y = r + dropout(F(x) + adapter(dropout(x))) and the gradients of <g, y> by the adapter's A and B and by
    the adapter's share of x, each stage against its definition on the stage's own inputs."""
    import torch
    rows, d = 320, 256
    inp = wl.make_inputs(wl.Workload("step", wl.LayerShape(d, 1024, 8, 2, 2, dtype), (rows,), seed=4))
    layer = parity.gpu_layer(inp.layers[0], rows)
    s = make(dtype, rows, 1, 8, d, d, ids=None, seed=3, dy=True)
    s["x"] = parity.to_device(inp.x, dtype)
    d_in, d_out = Dropout(0.05, 1234, 0), Dropout(0.1, 1234, 1)
    s["base"] = layer.forward(s["x"])
    h, z = binding.adapter_forward(s["x"], s["a"], s["b"], None, s["scale"], base=s["base"], dropout=d_in, want_z=True)
    check_forward(s, dtype, h, z, d_in)
    resid, g = s["x"], s["dy"]
    y = binding.dropout(h, d_out, residual=resid)
    want = ao.dropout(_host(h), 0.1, 1234, 1, residual=_host(resid))
    assert (np.abs(_host(y) - want) <= _eps(dtype) / 2 * np.abs(want) + 2.0**-21 * (1.2 * np.abs(_host(h)) + np.abs(_host(resid)))).all()
    dh = binding.dropout(g, d_out)
    s["dy"] = dh
    got = binding.adapter_backward(dh, s["x"], z, s["a"], s["b"], None, s["scale"], dx_base=s["dx_base"], dropout=d_in)
    check_backward(s, dtype, got, z, d_in)
    # the mask inside the adapter is the stand-alone one: on x with its dropout applied (and rounded, in bf16), no mask gives the same z
    xd = binding.dropout(s["x"], d_in)
    _, z2 = binding.adapter_forward(xd, s["a"], s["b"], None, s["scale"], want_z=True)
    zmag = np.abs(_host(xd)) @ np.abs(_host(s["a"])[0]).T
    assert (np.abs(_host(z) - _host(z2)) <= (_eps(dtype) / 2 + 2 * _chain(d, dtype) + 2.0**-22) * 1.01 * zmag).all()
    layer.destroy()
