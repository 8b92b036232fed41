"""moe_norm_* check their arguments on the host before anything is launched (no GPU needed here)."""
import ctypes
import math

import pytest

from paper_2411_10003_amd import binding

vp = ctypes.c_void_p
P = vp(0x1000)


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _cfg(rows=4, d=64, dtype=1, eps=1e-5):
    return binding._Norm(rows, d, dtype, eps)


def test_forward(lib):
    def call(c, X=P, R=None, gamma=P, beta=None, S=None, Y=P, mean=None, rstd=None):
        return lib.moe_norm_fwd(ctypes.byref(c) if c is not None else None, X, R, gamma, beta, S, Y, mean, rstd, None)

    assert call(None) == -1
    assert call(_cfg(), X=None) == -1 and call(_cfg(), gamma=None) == -1 and call(_cfg(), Y=None) == -1
    assert call(_cfg(), R=P) == -1 and call(_cfg(), S=P) == -1             # the residual and its sum: both or neither
    assert call(_cfg(), mean=P) == -1 and call(_cfg(), rstd=P) == -1
    for bad in (dict(rows=-1), dict(rows=1 << 30), dict(d=0), dict(d=16385), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan)):
        assert call(_cfg(**bad)) == -2, bad
    assert call(_cfg(dtype=5)) == -5
    assert call(_cfg(rows=0), X=None, gamma=None, Y=None) == 0             # nothing to do


def test_backward(lib):
    def call(c, dY=P, S=P, gamma=P, mean=P, rstd=P, dS=None, dX=P, dgamma=P, dbeta=None, ws=P):
        return lib.moe_norm_bwd(ctypes.byref(c) if c is not None else None, dY, S, gamma, mean, rstd, dS, dX, dgamma, dbeta, ws, None)

    assert call(None) == -1
    for missing in ("dY", "S", "gamma", "mean", "rstd", "dX", "dgamma"):
        assert call(_cfg(), **{missing: None}) == -1, missing
    assert call(_cfg(rows=0), dgamma=None) == -1                           # it is written without rows, too
    assert call(_cfg(), ws=None) == -4 and call(_cfg(), ws=vp(0x1010)) == -4
    assert call(_cfg(d=16385)) == -2 and call(_cfg(dtype=3)) == -5


def test_workspace(lib):
    n = ctypes.c_size_t()
    assert lib.moe_norm_workspace_bytes(ctypes.byref(_cfg(d=100)), ctypes.byref(n)) == 0
    assert n.value % 256 == 0 and n.value >= 100 * 8
    assert lib.moe_norm_workspace_bytes(ctypes.byref(_cfg(d=100)), None) == -1
    assert lib.moe_norm_workspace_bytes(ctypes.byref(_cfg(d=-1)), ctypes.byref(n)) == -2
