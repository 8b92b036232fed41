"""moe_muon_* check their arguments on the host before anything is launched (no GPU needed here)."""
import ctypes
import math

import pytest

from paper_2411_10003_amd import binding

vp = ctypes.c_void_p
GOOD = dict(n_tensors=2, count=3, rows=64, cols=256, transposed=(0, 1), dtype=1, nesterov=1, steps=5, momentum=0.95, eps=1e-7, a=3.4445, b=-4.775, c=2.0315,
            lr=0.02, weight_decay=0.1, scale=1.0)


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _cfg(**kw):
    f = {**GOOD, **kw}
    f["transposed"] = (ctypes.c_int * 8)(*f["transposed"])
    return binding._Muon(*(f[n] for n, _ in binding._Muon._fields_))


BAD = [dict(n_tensors=0), dict(n_tensors=9), dict(count=0), dict(count=32768), dict(rows=0), dict(cols=0), dict(rows=65537), dict(rows=32768, cols=32768), dict(transposed=(0, 2)),
       dict(nesterov=2), dict(steps=0), dict(steps=17), dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=math.nan), dict(eps=0.0), dict(eps=math.inf),
       dict(a=17.0), dict(b=math.nan), dict(c=-math.inf), dict(lr=math.inf), dict(weight_decay=math.nan), dict(scale=math.inf)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_sizes_and_constants(lib, bad):
    n = ctypes.c_size_t()
    two = (vp * 2)(0x1000, 0x2000)
    assert lib.moe_muon_workspace_bytes(ctypes.byref(_cfg(**bad)), ctypes.byref(n)) == -2
    assert lib.moe_muon_step(ctypes.byref(_cfg(**bad)), two, two, two, None, None, vp(0x1000), None) == -2


def test_pointers(lib):
    n = ctypes.c_size_t()
    two, missing, c = (vp * 2)(0x1000, 0x2000), (vp * 2)(0x1000, 0), _cfg()
    ws = vp(0x1000)
    assert lib.moe_muon_workspace_bytes(None, ctypes.byref(n)) == -1 and lib.moe_muon_workspace_bytes(ctypes.byref(c), None) == -1
    assert lib.moe_muon_step(None, two, two, two, None, None, ws, None) == -1
    for k in range(3):
        for bad in (None, missing):
            args = [two, two, two]
            args[k] = bad
            assert lib.moe_muon_step(ctypes.byref(c), *args, None, None, ws, None) == -1
    assert lib.moe_muon_step(ctypes.byref(c), two, two, two, two, None, ws, None) == -5        # copies of bf16 weights
    assert lib.moe_muon_step(ctypes.byref(c), two, two, two, None, None, None, None) == -4
    assert lib.moe_muon_step(ctypes.byref(c), two, two, two, None, None, vp(0x1080), None) == -4
    assert lib.moe_muon_workspace_bytes(ctypes.byref(_cfg(dtype=2)), ctypes.byref(n)) == -5


def test_workspace(lib):
    """Enough for the iterates of every matrix, padded to multiples of 64, in one plane for bf16 weights and two for fp32."""
    n = ctypes.c_size_t()
    for dtype, planes in ((1, 1), (0, 2)):
        assert lib.moe_muon_workspace_bytes(ctypes.byref(_cfg(rows=100, cols=70, dtype=dtype)), ctypes.byref(n)) == 0
        assert n.value % 256 == 0 and n.value >= 6 * 128 * 128 * 2 * planes
