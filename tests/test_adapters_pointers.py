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
