"""CPU-only: pointers that the adapters' calls refuse on the host.  No pointer here is ever read."""
import ctypes as C

import pytest

from paper_2502_04416_b200 import binding, build

P = 1 << 20                                                 # an aligned address that nobody reads
NAMES = ("dy", "x", "z", "base", "out", "ids", "a", "b", "scale", "ga", "gb", "scratch")
AT = {name: (i + 1) * P for i, name in enumerate(NAMES)}    # all apart
ROWS, N, R, D_IN, D_OUT = 300, 3, 8, 64, 32


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _set(p):
    return binding.CmoeAdapters(N, R, D_IN, D_OUT, 0, p["a"], p["b"], p["scale"])


def _fwd(lib, rows=ROWS, ld=None, **kw):
    p, ld = {**AT, **kw}, {**dict(x=D_IN, base=D_OUT, out=D_OUT), **(ld or {})}
    return lib.cmoe_adapter_forward(C.byref(_set(p)), p["x"], ld["x"], p["ids"], rows, None, p["base"], ld["base"], p["out"], ld["out"], p["z"],
                                    p["scratch"], 1 << 19, None)


def _bwd(lib, rows=ROWS, ld=None, **kw):
    p, ld = {**AT, **kw}, {**dict(dy=D_OUT, x=D_IN, base=D_IN, out=D_IN), **(ld or {})}
    return lib.cmoe_adapter_backward(C.byref(_set(p)), p["dy"], ld["dy"], p["x"], ld["x"], p["z"], p["ids"], rows, None, p["base"], ld["base"],
                                     p["out"], ld["out"], p["ga"], p["gb"], p["scratch"], 1 << 19, None)


@pytest.mark.parametrize("rows", [1, 300])
@pytest.mark.parametrize("by", [1, 2, 3])
def test_row_numbers_off_their_boundary(lib, rows, by):
    """A misaligned address would fault on the device."""
    assert _fwd(lib, rows, ids=AT["ids"] + by) == -1 and b"row_adapter" in lib.cmoe_last_error()
    assert _bwd(lib, rows, ids=AT["ids"] + by) == -1 and b"row_adapter" in lib.cmoe_last_error()


# ------------------------------------------------------------------ overlaps
BYTES = dict(dy=ROWS * D_OUT * 2, x=ROWS * D_IN * 2, z=ROWS * R * 4, base=ROWS * D_IN * 2, out=ROWS * D_IN * 2, ids=ROWS * 4, a=N * R * D_IN * 2,
             b=N * R * D_OUT * 2, scale=N * 4, ga=N * R * D_IN * 2, gb=N * R * D_OUT * 2, scratch=1 << 16)


def _apart(lib, call, moved, to):
    """Whether the call takes `moved` at the end of `to` and refuses it one boundary earlier.  A call that is taken would be launched, so
    that is asked of one which is refused later, for a scratch that is named last."""
    size = dict(BYTES, base=ROWS * D_OUT * 2, out=ROWS * D_OUT * 2) if call is _fwd else BYTES
    step = 256 if moved == "scratch" else 16
    inside = AT[to] + (size[to] - 1) // step * step
    assert call(lib, **{moved: inside}) == -1, (moved, to)
    text = lib.cmoe_last_error().decode()
    assert "overlap" in text, text
    return text


@pytest.mark.parametrize("moved,others", [("z", ("x", "base", "out", "ids", "a", "b", "scale")),
                                          ("scratch", ("x", "base", "out", "ids", "a", "b", "scale", "z")),
                                          ("out", ("ids", "a", "b", "scale"))])
def test_forward_overlaps(lib, moved, others):
    for to in others:
        text = _apart(lib, _fwd, moved, to)
        assert {"ids": "row_adapter"}.get(to, to) in text and moved in text


@pytest.mark.parametrize("moved,others", [("ga", ("dy", "x", "z", "base", "out", "ids", "a", "b", "scale", "gb")),
                                          ("gb", ("dy", "x", "z", "base", "out", "ids", "a", "b", "scale", "ga")),
                                          ("scratch", ("dy", "x", "z", "base", "out", "ids", "a", "b", "scale", "ga", "gb")),
                                          ("out", ("z", "ids", "a", "b", "scale"))])
def test_backward_overlaps(lib, moved, others):
    names = dict(ids="row_adapter", ga="grad_a", gb="grad_b", base="dx_base", out="dx")
    for to in others:
        text = _apart(lib, _bwd, moved, to)
        assert names.get(to, to) in text and names.get(moved, moved) in text


def test_what_only_lies_side_by_side_does_not_overlap(lib):
    """z, a run of bytes, in the gap between a matrix's rows or behind its last one; the call is then refused for the overlap that the
    scratch has with a, which is looked at later."""
    def says(**kw):
        assert _fwd(lib, **{**dict(scratch=AT["a"]), **kw}) == -1
        return lib.cmoe_last_error().decode()
    size = ROWS * R * 4
    ld = size // 2 + 64 + D_IN                              # in elements of two bytes: rows with a gap that z fits in
    assert "scratch and a" in says()
    assert "scratch and a" in says(ld=dict(x=ld), z=AT["x"] + D_IN * 2)
    assert "z and x" in says(ld=dict(x=ld), z=AT["x"] + D_IN * 2 - 16)
    assert "z and x" in says(ld=dict(x=ld), z=AT["x"] + ld * 2 - size + 16)
    assert "scratch and a" in says(z=AT["x"] + ROWS * D_IN * 2)
    assert "z and x" in says(z=AT["x"] + ROWS * D_IN * 2 - 16)
    assert "z and x" in says(z=AT["x"] - size + 16)
    assert "scratch and a" in says(z=AT["x"] - size)


def test_what_is_not_read_may_lie_anywhere(lib):
    """Without the weights' gradients x and z are not looked at; with the gradients they are."""
    bad = dict(scratch=AT["a"])
    assert _bwd(lib, ga=None, gb=None, x=AT["out"], z=AT["out"], **bad) == -1 and b"scratch and a" in lib.cmoe_last_error()
    assert _bwd(lib, z=AT["out"], **bad) == -1 and b"scratch and a" in lib.cmoe_last_error()
    assert _bwd(lib, z=AT["out"]) == -1 and b"dx and z" in lib.cmoe_last_error()


@pytest.mark.parametrize("what", ["x", "residual", "out"])
@pytest.mark.parametrize("rows,ld", [(2**31 - 1, 2**40), (2**30, 2**31), (2**25, 2**36)])
def test_dropout_of_more_than_all_memory(lib, what, rows, ld):
    """Products of rows and strides that pass 64 bits, or come near: the check for overlaps counts with them."""
    lds = {**dict(x=10, residual=10, out=10), what: ld}
    drop = binding.CmoeDropoutConfig(0.1, 1, 0, 0)
    at = dict(x=1 << 44, residual=1 << 45, out=1 << 46)
    assert lib.cmoe_dropout(at["x"], lds["x"], at["residual"], lds["residual"], rows, 10, 1, C.byref(drop), at["out"], lds["out"], None) == -1
    assert b"stride" in lib.cmoe_last_error()
