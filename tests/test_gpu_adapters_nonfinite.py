"""-m gpu: infinities and NaN in the rows of an adapter, in the gradients of its own weights, against sums formed term by term in 64 bits.

All finite values are small whole numbers, so sums are exact in 32 bits and a result is off by its one rounding (eps / 2).  The narrow
operands (e and z) are whole numbers of at most eight bits, infinities or NaN: in bf16 calls, where they enter the sums in two parts, what
multiplies an infinity has to be no zero unless the value is one."""
import numpy as np
import pytest

from paper_2502_04416_b200 import binding

pytestmark = pytest.mark.gpu

SHAPES = [  # type, rows, adapters, rank, row_adapter given
    ("bf16", 40, 3, 8, True), ("bf16", 40, 1, 16, False), ("bf16", 300, 3, 24, True), ("bf16", 300, 2, 32, True), ("bf16", 700, 3, 64, True),
    ("bf16", 1100, 3, 48, True), ("bf16", 1100, 1, 64, False), ("bf16", 4200, 3, 24, True),          # tiles of 128 rows
    ("fp32", 40, 3, 8, True), ("fp32", 300, 2, 40, True)]


def _whole(rng, shape, most):
    """Whole numbers from 1 to most, of either sign."""
    return rng.integers(1, most + 1, shape) * rng.choice([-1, 1], shape) * 1.0


@pytest.mark.parametrize("dtype,rows,n,r,with_ids", SHAPES)
@pytest.mark.parametrize("where", ["x", "dy", "z"])
def test_sums_over_rows_with_infinities(dtype, rows, n, r, with_ids, where):
    import torch
    d_in, d_out = 72, 136
    rng = np.random.default_rng(rows + r)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    v = dict(x=_whole(rng, (rows, d_in), 3), dy=np.zeros((rows, d_out)), z=_whole(rng, (rows, r), 3),
             a=_whole(rng, (n, r, d_in), 2), b=_whole(rng, (n, d_out, r), 2))
    v["dy"][np.arange(rows), rng.integers(0, d_out, rows)] = _whole(rng, rows, 3)                    # e = b dy: eight bits hold it
    v["dy"][np.arange(rows), rng.integers(0, d_out, rows)] = _whole(rng, rows, 3)
    ids = rng.integers(0, n, rows) if with_ids else np.zeros(rows, dtype=np.int64)
    few = rng.choice(rows, 6, replace=False)
    for i, t in enumerate(few):
        at = rng.integers(0, v[where].shape[1])
        v[where][t, at] = [np.inf, -np.inf, np.inf, -np.inf, np.nan, np.inf][i]
    dev = {k: torch.from_numpy(t).cuda().to(dt if k != "z" else torch.float32) for k, t in v.items()}
    got = binding.adapter_backward(dev["dy"], dev["x"], dev["z"], dev["a"], dev["b"],
                                   torch.from_numpy(ids.astype(np.int32)).cuda() if with_ids else None)
    want = [np.zeros((rows, d_in)), np.zeros((n, r, d_in)), np.zeros((n, d_out, r))]
    with np.errstate(invalid="ignore"):
        for t, k in enumerate(ids):
            e = (v["b"][k] * v["dy"][t][:, None]).sum(0)
            want[0][t] = (v["a"][k] * e[:, None]).sum(0)
            want[1][k] += e[:, None] * v["x"][t][None, :]
            want[2][k] += v["dy"][t][:, None] * v["z"][t][None, :]
        assert any(np.isinf(w).any() for w in want)
        for g, w in zip(got, want):
            g = g.double().cpu().numpy()
            np.testing.assert_array_equal(np.isnan(g), np.isnan(w))
            np.testing.assert_array_equal(g[np.isinf(w)], w[np.isinf(w)])
            ok = np.isfinite(w)
            assert (np.abs(g[ok] - w[ok]) <= torch.finfo(dt).eps / 2 * np.abs(w[ok])).all()


@pytest.mark.parametrize("rows,r", [(40, 8), (300, 64), (1100, 64), (4200, 24)])
def test_every_nan_of_z_is_one(rows, r):
    """A NaN is a NaN whatever its bits: the one whose payload lies in the 16 low bits of the 32 too."""
    import torch
    g = torch.Generator("cuda").manual_seed(0)
    x, dy = (torch.randn(rows, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    a, b = torch.randn(1, r, 64, generator=g, device="cuda").bfloat16(), torch.randn(1, 64, r, generator=g, device="cuda").bfloat16()
    z = torch.randn(rows, r, generator=g, device="cuda")
    z.view(torch.int32)[rows // 2, 5] = 0x7F800001
    _, ga, gb = binding.adapter_backward(dy, x, z, a, b)
    assert gb[0, :, 5].isnan().all() and not ga.isnan().any()
    rest = [i for i in range(r) if i != 5]
    assert not gb[0][:, rest].isnan().any()


@pytest.mark.parametrize("dtype,rows,n,r,with_ids", SHAPES + [("bf16", 1, 1, 8, False), ("fp32", 1100, 3, 64, True)])
@pytest.mark.parametrize("where", ["x", "base"])
def test_a_rows_own_infinities(dtype, rows, n, r, with_ids, where):
    """The forward: an infinity or a NaN of a row goes through both products as the formulas have it, into z and out."""
    import torch
    d_in, d_out = 72, 136
    rng = np.random.default_rng(rows + r)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    v = dict(x=np.zeros((rows, d_in)), a=_whole(rng, (n, r, d_in), 2), b=_whole(rng, (n, d_out, r), 2), base=_whole(rng, (rows, d_out), 3))
    v["x"][np.arange(rows), rng.integers(0, d_in, rows)] = _whole(rng, rows, 3)
    ids = rng.integers(0, n, rows) if with_ids else np.zeros(rows, dtype=np.int64)
    for i, t in enumerate(rng.choice(rows, min(rows, 6), replace=False)):
        v[where][t, rng.integers(0, v[where].shape[1])] = [np.inf, -np.inf, np.inf, -np.inf, np.nan, np.inf][i]
    v["b"][:, ::3] = np.abs(v["b"][:, ::3])                  # some columns where no two infinities of other signs meet
    v["a"] = np.abs(v["a"])
    dev = {k: torch.from_numpy(t).cuda().to(dt) for k, t in v.items()}
    out, z = binding.adapter_forward(dev["x"], dev["a"], dev["b"], torch.from_numpy(ids.astype(np.int32)).cuda() if with_ids else None,
                                     base=dev["base"], want_z=True)
    with np.errstate(invalid="ignore"):
        want_z = np.stack([(v["a"][k] * v["x"][t]).sum(1) for t, k in enumerate(ids)])
        want = np.stack([v["base"][t] + (v["b"][k] * want_z[t]).sum(1) for t, k in enumerate(ids)])
        assert np.isinf(want).any()
        for g, w, half in ((out, want, torch.finfo(dt).eps / 2), (z, want_z, 0.0)):
            g = g.double().cpu().numpy()
            np.testing.assert_array_equal(np.isnan(g), np.isnan(w))
            np.testing.assert_array_equal(g[np.isinf(w)], w[np.isinf(w)])
            ok = np.isfinite(w)
            assert (np.abs(g[ok] - w[ok]) <= half * np.abs(w[ok])).all()
