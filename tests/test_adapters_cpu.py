"""CPU-only: pins of the adapter and dropout oracle, and every refusal of the C-ABI calls that is decided on the host."""
import ctypes as C
import itertools

import numpy as np
import pytest

from oracle import adapters_oracle as ao
from paper_2502_04416_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


# ------------------------------------------------------------------ the generator
def test_philox_known_answers():
    """The published known-answer vectors of Philox 4x32-10."""
    for ctr, key, want in [
        ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
        ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
        ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
    ]:
        assert tuple(ao.philox(np.array(ctr, dtype=np.uint32), key)) == want


def test_mask_by_hand():
    """Column 8 c + j of row t: half j of the block on (c, t, offset) under the seed."""
    seed, offset, row0 = 0x123456789ABCDEF0, 0x1_0000_0005, 2**32 - 3
    mask = ao.keep_mask(3, 21, 0.3, seed, offset, row0)
    thr = int(0.3 * 65536 + 0.5)
    for t, col in itertools.product(range(3), range(21)):
        w = ao.philox(np.array([col // 8, (row0 + t) % 2**32, 5, 1], dtype=np.uint32), (0x9ABCDEF0, 0x12345678))
        half = (int(w[(col % 8) // 2]) >> (16 * (col % 2))) & 0xFFFF
        assert mask[t, col] == (half >= thr)


def test_mask_rate_and_independence():
    m = ao.keep_mask(400, 1000, 0.25, 7)
    n = m.size                                              # binomial: six standard deviations
    assert abs(m.mean() - 0.75) < 6 * np.sqrt(0.75 * 0.25 / n)
    other = [ao.keep_mask(400, 1000, 0.25, 8), ao.keep_mask(400, 1000, 0.25, 7, offset=1), ao.keep_mask(400, 1000, 0.25, 7, row0=400)]
    for o in other:                                         # agreement of independent masks: 0.75^2 + 0.25^2
        assert abs((m == o).mean() - 0.625) < 6 * np.sqrt(0.625 * 0.375 / n)
    assert np.array_equal(ao.keep_mask(150, 1000, 0.25, 7, row0=250), m[250:])
    assert ao.keep_mask(5, 9, 0.0, 3).all()


# ------------------------------------------------------------------ the adapters' formulas
def _small(rng, rows=5, n=2, r=8, d_in=16, d_out=24):
    return dict(x=rng.normal(size=(rows, d_in)), a=rng.normal(size=(n, r, d_in)), b=rng.normal(size=(n, d_out, r)),
                scale=rng.uniform(0.5, 2, n), base=rng.normal(size=(rows, d_out)))


def test_forward_special_cases():
    rng = np.random.default_rng(0)
    s = _small(rng)
    ids = np.array([0, 1, -1, 2, 0])                        # -1 and n: no adapter
    out, z = ao.adapter_forward(s["x"], s["a"], s["b"], ids, s["scale"], s["base"])
    np.testing.assert_array_equal(out[2:4], s["base"][2:4])
    np.testing.assert_array_equal(z[2:4], 0)
    for t in (0, 1, 4):                                     # the merged weight W + s B A gives the same rows
        merged = s["scale"][ids[t]] * s["b"][ids[t]] @ s["a"][ids[t]]
        np.testing.assert_allclose(out[t], s["base"][t] + merged @ s["x"][t], rtol=1e-12, atol=1e-12)
    zero, _ = ao.adapter_forward(s["x"], s["a"], 0 * s["b"], ids, s["scale"], s["base"])
    np.testing.assert_array_equal(zero, s["base"])          # B = 0, as adapters start: the projection itself


def test_gradients_against_differences():
    """The loss <dy, out> is linear in x, A and B one at a time: central differences are exact up to rounding."""
    rng = np.random.default_rng(1)
    s = _small(rng)
    ids = np.array([1, 0, -1, 1, 1])
    keep = ao.keep_mask(5, 16, 0.3, 11)
    mask = keep * (65536 / (65536 - ao.threshold(0.3)))
    dy = rng.normal(size=s["base"].shape)

    def loss(x, a, b):
        return float((dy * ao.adapter_forward(x * mask, a, b, ids, s["scale"], s["base"])[0]).sum())

    _, z = ao.adapter_forward(s["x"] * mask, s["a"], s["b"], ids, s["scale"])
    dx, ga, gb = ao.adapter_backward(dy, s["x"] * mask, z, s["a"], s["b"], ids, s["scale"], mask)
    for name, grad in (("x", dx), ("a", ga), ("b", gb)):
        for _ in range(40):
            at = tuple(rng.integers(0, n) for n in grad.shape)
            hi, lo = ({k: v.copy() for k, v in s.items() if k in "xab"} for _ in range(2))
            hi[name][at] += 0.5
            lo[name][at] -= 0.5
            assert abs(loss(hi["x"], hi["a"], hi["b"]) - loss(lo["x"], lo["a"], lo["b"]) - grad[at]) < 1e-10 * (1 + abs(grad[at])) * 100
    base = rng.normal(size=dx.shape)
    np.testing.assert_allclose(ao.adapter_backward(dy, s["x"] * mask, z, s["a"], s["b"], ids, s["scale"], mask, base)[0], dx + base)
    assert (dx[2] == 0).all() and (dx[~keep] == 0).all()


# ------------------------------------------------------------------ refusals (no pointer is ever dereferenced)
P = 1 << 20                                                 # an aligned address that nobody reads


def _ad(**kw):
    d = dict(n_adapters=4, rank=8, d_in=64, d_out=32, dtype=0, a=P, b=P, scale=None)
    return binding.CmoeAdapters(*[{**d, **kw}[k] for k in ("n_adapters", "rank", "d_in", "d_out", "dtype", "a", "b", "scale")])


def _drop(**kw):
    d = dict(p=0.1, seed=1, offset=0, row0=0)
    return binding.CmoeDropoutConfig(*[{**d, **kw}[k] for k in ("p", "seed", "offset", "row0")])


def _fwd(lib, ad=None, x=P, ldx=64, ids=None, rows=4, drop=None, base=2 * P, ld_base=32, out=3 * P, ld_out=32, z=None, scratch=None, nbytes=0):
    ad = _ad() if ad is None else ad
    return lib.cmoe_adapter_forward(C.byref(ad), x, ldx, ids, rows, C.byref(drop) if drop else None, base, ld_base, out, ld_out, z,
                                    scratch, nbytes, None)


def _bwd(lib, ad=None, dy=P, ld_dy=32, x=2 * P, ldx=64, z=3 * P, ids=None, rows=4, drop=None, base=None, ld_base=0, dx=4 * P, ld_dx=64,
         ga=5 * P, gb=6 * P, scratch=7 * P, nbytes=1 << 30):
    ad = _ad() if ad is None else ad
    return lib.cmoe_adapter_backward(C.byref(ad), dy, ld_dy, x, ldx, z, ids, rows, C.byref(drop) if drop else None, base, ld_base, dx, ld_dx,
                                     ga, gb, scratch, nbytes, None)


@pytest.mark.parametrize("kw", [dict(n_adapters=0), dict(n_adapters=1025), dict(rank=0), dict(rank=4), dict(rank=12), dict(rank=72),
                                dict(d_in=0), dict(d_in=60), dict(d_out=20), dict(d_out=-8), dict(d_in=(1 << 24) + 8), dict(dtype=2),
                                dict(a=None), dict(b=None), dict(a=P + 8), dict(b=P + 2), dict(scale=P + 4)])
def test_adapter_set_refusals(lib, kw):
    assert _fwd(lib, _ad(**kw)) == -1
    assert _bwd(lib, _ad(**kw)) == -1
    if not {"a", "b", "scale"} & set(kw):
        assert lib.cmoe_adapter_scratch_bytes(C.byref(_ad(**kw)), 1000, 1, 1) == 0


@pytest.mark.parametrize("kw", [dict(x=None), dict(out=None), dict(rows=-1), dict(x=P + 8), dict(out=P + 4), dict(base=P + 2),
                                dict(ldx=56), dict(ldx=68), dict(ld_out=24), dict(ld_out=36), dict(ld_base=16),
                                dict(out=P), dict(out=P + 48, ld_out=64), dict(base=3 * P + 16, ld_base=32),
                                dict(base=3 * P, ld_base=40), dict(z=P + 4),
                                dict(ids=P, rows=257), dict(ids=P, rows=257, scratch=P + 128, nbytes=1 << 30),
                                dict(drop=_drop(p=-0.1)), dict(drop=_drop(p=1.0)), dict(drop=_drop(p=float("nan"))),
                                dict(drop=_drop(p=1 - 2.0**-18)), dict(drop=_drop(row0=-1)), dict(drop=_drop(row0=2**32 - 3))])
def test_forward_refusals(lib, kw):
    assert _fwd(lib, **kw) == -1


@pytest.mark.parametrize("kw", [dict(dy=None), dict(x=None), dict(z=None), dict(ga=None), dict(gb=None), dict(ga=None, gb=None, dx=None),
                                dict(ga=P + 2), dict(dx=P), dict(dx=2 * P), dict(base=4 * P + 16, ld_base=64), dict(base=P + 8, ld_base=64),
                                dict(ld_dx=56), dict(ld_dy=16), dict(ldx=32), dict(rows=-2), dict(scratch=None), dict(scratch=P + 16),
                                dict(drop=_drop(p=1.5))])
def test_backward_refusals(lib, kw):
    assert _bwd(lib, **kw) == -1


def test_capacity_refusals(lib):
    need = lib.cmoe_adapter_scratch_bytes(C.byref(_ad()), 257, 1, 0)
    assert need > 0 and _fwd(lib, ids=P, rows=257, scratch=P, nbytes=need - 1) == -4
    need = lib.cmoe_adapter_scratch_bytes(C.byref(_ad()), 4, 0, 1)
    assert need > 0 and _bwd(lib, nbytes=need - 1) == -4
    assert _fwd(lib, rows=2**30 + 1) == -4 and _bwd(lib, rows=2**30 + 1) == -4
    assert lib.cmoe_adapter_scratch_bytes(C.byref(_ad()), 256, 1, 0) == 0       # such a batch finds its tiles without
    assert lib.cmoe_adapter_scratch_bytes(C.byref(_ad()), 100000, 0, 0) == 0    # one adapter for every row
    assert b"scratch" in lib.cmoe_last_error() or lib.cmoe_last_error()


@pytest.mark.parametrize("bf", [0, 1])
def test_scratch_holds_the_worst_case(lib, bf):
    """Tiles of at least 32 rows: every adapter and the rows without one may leave a tile part filled."""
    for rows, n, r in itertools.product((1, 31, 257, 5000), (1, 7, 1024), (8, 16, 32, 64)):
        m = 32
        groups = min(n + 1, rows)
        tiles = max((rows - groups + 1 + m - 1) // m + groups - 1, 1)            # one large group, the others a row each
        ad = _ad(n_adapters=n, rank=r, dtype=bf)
        per = m * (-(-r // 8) * 8 * 4 if bf else (8 if r <= 8 else 16 if r <= 16 else 32 if r <= 32 else 64) * 4)
        have = lib.cmoe_adapter_scratch_bytes(C.byref(ad), rows, 1, 1)
        assert have >= (n + 2) * 4 + tiles * 4 + tiles * m * 4 + 2 * tiles * per


def test_empty_calls_are_no_ops(lib):
    assert _fwd(lib, rows=0) == 0
    assert _fwd(lib, rows=0, x=None, out=None) == 0
    assert lib.cmoe_dropout(None, 0, None, 0, 0, 5, 0, C.byref(_drop()), None, 0, None) == 0
    assert lib.cmoe_dropout(None, 0, None, 0, 5, 0, 1, C.byref(_drop()), None, 0, None) == 0


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(cols=-1), dict(dtype=7), dict(drop=None), dict(x=None), dict(out=None), dict(ldx=9),
                                dict(ldo=8), dict(res=2 * P, ldr=9), dict(x=P + 1), dict(out=3 * P + 1), dict(out=P + 2), dict(out=P, ldo=12),
                                dict(res=3 * P + 4, ldr=10), dict(drop=_drop(p=1.0)), dict(drop=_drop(p=-1e-9)), dict(drop=_drop(row0=2**32))])
def test_dropout_refusals(lib, kw):
    d = {**dict(x=P, ldx=10, res=None, ldr=0, rows=6, cols=10, dtype=0, drop=_drop(), out=3 * P, ldo=10), **kw}
    st = lib.cmoe_dropout(d["x"], d["ldx"], d["res"], d["ldr"], d["rows"], d["cols"], d["dtype"], C.byref(d["drop"]) if d["drop"] else None,
                          d["out"], d["ldo"], None)
    assert st == -1


def test_column_slices_of_one_matrix_do_not_overlap(lib):
    """x, base and out as column slices of one wider matrix pass that check: the call is refused for its scratch, which is looked
    at later."""
    def says(**kw):
        assert _fwd(lib, ids=P, rows=257, scratch=None, **kw) == -1
        return lib.cmoe_last_error().decode()
    assert "scratch" in says(x=P, ldx=96, out=P + 128, ld_out=96, base=None)
    assert "scratch" in says(x=P, ldx=128, out=P + 128, ld_out=128, base=P + 192, ld_base=128)
    assert "scratch" in says(x=P + 64, ldx=96, out=P, ld_out=96, base=P, ld_base=96)         # out is base
    assert "x and out" in says(x=P, ldx=96, out=P + 112, ld_out=96, base=None)
    assert "x and out" in says(x=P, ldx=96, out=P + 144, ld_out=96, base=None)               # runs into the next row
    assert "base and out" in says(x=P, ldx=128, out=P + 128, ld_out=128, base=P + 176, ld_base=128)


def test_adapted_forward_refusals(lib):
    assert lib.cmoe_ffn_forward_adapted(None, P, 1, C.byref(_ad()), None, 2 * P, None, 0, None) == -1


def test_scratch_grows_with_the_batch_and_holds_tall_tiles(lib):
    """A workspace for the longest batch serves the shorter ones, whatever tiles they take; tiles of 128 rows are counted whole."""
    for n, r, backward in itertools.product((1, 5, 32, 64), (8, 24, 32, 40, 64), (0, 1)):
        ad = _ad(n_adapters=n, rank=r)
        sizes = [lib.cmoe_adapter_scratch_bytes(C.byref(ad), rows, 1, backward) for rows in range(300, 9000, 37)]
        assert sizes == sorted(sizes)
        for rows in (1024, 2049, 4096, 8191):
            if r > 16 and rows >= max(64 * n, 4096 if r <= 32 else 1024):
                tiles = (rows - min(n + 1, rows) + 1 + 127) // 128 + n           # one large group, the others a row each
                u = 2 * tiles * 128 * (128 if r <= 32 else 256) if backward else 0
                assert lib.cmoe_adapter_scratch_bytes(C.byref(ad), rows, 1, backward) >= (n + 2) * 4 + tiles * 4 + tiles * 128 * 4 + u
