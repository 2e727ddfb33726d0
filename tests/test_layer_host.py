"""Host checks of the position-wise entry points: bad arguments are refused
before any launch (no GPU: every call here returns from those checks)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO
from paper_2608_00938_amd import grace as G

needs_lib = pytest.mark.skipif(not os.path.exists(G._LIB_PATH), reason="libgrace.so not built")


def at(k):
    """A device address that is never read: 16 MiB apart."""
    return ctypes.c_void_p(k << 24)


def norm(**kw):
    a = dict(x=at(1), res=at(2), w=at(3), R=4, D=64, eps=1e-6, dtype=G.GRACE_BF16, to=G.GRACE_BF16,
             sum=at(4), out=at(5), scale=at(6))
    a.update(kw)
    return G.library().grace_rms_norm(a["x"], a["res"], a["w"], a["R"], a["D"], a["eps"], a["dtype"],
                                      a["to"], a["sum"], a["out"], a["scale"], None)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), G.GRACE_ERR_UNSUPPORTED), (dict(dtype=-1), G.GRACE_ERR_UNSUPPORTED),
    (dict(to=3), G.GRACE_ERR_UNSUPPORTED), (dict(R=-1), G.GRACE_ERR_SHAPE),
    (dict(D=0), G.GRACE_ERR_SHAPE), (dict(D=32769), G.GRACE_ERR_SHAPE),
    (dict(eps=0.0), G.GRACE_ERR_SHAPE), (dict(eps=math.nan), G.GRACE_ERR_SHAPE),
    (dict(eps=math.inf), G.GRACE_ERR_SHAPE), (dict(x=None), G.GRACE_ERR_NULL),
    (dict(w=None), G.GRACE_ERR_NULL), (dict(out=None), G.GRACE_ERR_NULL),
    (dict(to=G.GRACE_E4M3, scale=None), G.GRACE_ERR_NULL),
    (dict(out=at(1)), G.GRACE_ERR_ALIAS), (dict(out=at(2)), G.GRACE_ERR_ALIAS),
    (dict(out=at(4)), G.GRACE_ERR_ALIAS), (dict(sum=at(3)), G.GRACE_ERR_ALIAS),
    (dict(sum=ctypes.c_void_p((1 << 24) + 64)), G.GRACE_ERR_ALIAS),       # inside x, not x itself
    (dict(to=G.GRACE_E4M3, scale=at(5)), G.GRACE_ERR_ALIAS),
    (dict(to=G.GRACE_E4M3, scale=at(4)), G.GRACE_ERR_ALIAS),
    # sum may be x, and then still not partly residual
    (dict(sum=at(1), res=ctypes.c_void_p((1 << 24) + 64)), G.GRACE_ERR_ALIAS),
    (dict(R=2 ** 31 - 1, D=32768), G.GRACE_ERR_ALIAS),                    # sizes in 64 bits
    (dict(R=0, x=None, out=None), G.GRACE_OK),
])
def test_norm_rejects(kw, status):
    assert norm(**kw) == status


@needs_lib
def test_norm_max_d():
    assert G.grace_rms_norm_max_d() == 32768


def test_norm_binding_checks_every_tensor(monkeypatch):
    """Shapes, types and layouts that the sizes passed on would not fit are
    refused before the library is reached."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(G, "library", Library)
    x, w = torch.zeros(4, 64), torch.zeros(64)
    for kw in (dict(weight=torch.zeros(63)), dict(residual=torch.zeros(4, 63)), dict(sum_out=torch.zeros(3, 64)),
               dict(out=torch.zeros(4, 65)), dict(x=torch.zeros(64, 4).t()),
               dict(out=torch.zeros(4, 64).to(torch.float8_e4m3fn), out_scale=torch.zeros(3))):
        with pytest.raises(ValueError):
            G.grace_rms_norm(**{**dict(x=x, weight=w), **kw})
    for kw in (dict(weight=w.bfloat16()), dict(residual=x.bfloat16()), dict(sum_out=x.double()),
               dict(x=x.half()), dict(out_dtype=torch.float16), dict(out_dtype=torch.float64)):
        with pytest.raises(TypeError):
            G.grace_rms_norm(**{**dict(x=x, weight=w), **kw})
    assert calls == []


def test_oracle_e4m3_grid():
    """Every e4m3 code is its own rounding, and half-way values go to the even code."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    codes = np.unique(codes[np.isfinite(codes)]).astype(np.float64)
    assert np.array_equal(LO.e4m3(codes), codes) and codes[-1] == LO.E4M3_MAX
    mid = (codes[:-1] + codes[1:]) / 2
    want = torch.from_numpy(mid).float().to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(LO.e4m3(mid), want)


def test_oracle_norm_closed_forms():
    h, y = LO.rms_norm(np.full((2, 8), 3.0), np.ones(8), 1e-300, residual=np.full((2, 8), -5.0))
    assert (h == -2).all() and np.allclose(y, -1, rtol=1e-15)
    _, y = LO.rms_norm(np.array([[3.0, 4.0]]), np.array([2.0, 1.0]), 0.5)
    assert np.allclose(y, np.array([[6.0, 4.0]]) / math.sqrt(13.0), rtol=1e-15)


def linear(**kw):
    a = dict(x=at(1), xs=at(2), w=at(3), ws=at(4), bias=at(5), res=at(6), R=8, N=16, K=32, act=0,
             dtype=G.GRACE_BF16, to=G.GRACE_BF16, out=at(7))
    a.update(kw)
    return G.library().grace_linear(a["x"], a["xs"], a["w"], a["ws"], a["bias"], a["res"], a["R"], a["N"],
                                    a["K"], a["act"], a["dtype"], a["to"], a["out"], None)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), G.GRACE_ERR_UNSUPPORTED), (dict(dtype=-1), G.GRACE_ERR_UNSUPPORTED),
    (dict(to=2), G.GRACE_ERR_UNSUPPORTED), (dict(act=4), G.GRACE_ERR_UNSUPPORTED),
    (dict(act=-1), G.GRACE_ERR_UNSUPPORTED), (dict(R=-1), G.GRACE_ERR_SHAPE),
    (dict(N=0), G.GRACE_ERR_SHAPE), (dict(K=0), G.GRACE_ERR_SHAPE),
    (dict(N=(1 << 30) + 1), G.GRACE_ERR_SHAPE), (dict(K=(1 << 30) + 1), G.GRACE_ERR_SHAPE),
    (dict(R=1 << 30, N=1 << 10), G.GRACE_ERR_SHAPE), (dict(R=1 << 30, K=1 << 10), G.GRACE_ERR_SHAPE),
    (dict(N=1 << 25, K=1 << 15), G.GRACE_ERR_SHAPE),
    (dict(x=None), G.GRACE_ERR_NULL), (dict(w=None), G.GRACE_ERR_NULL), (dict(out=None), G.GRACE_ERR_NULL),
    (dict(out=at(1)), G.GRACE_ERR_ALIAS), (dict(out=at(2)), G.GRACE_ERR_ALIAS),
    (dict(out=at(3)), G.GRACE_ERR_ALIAS), (dict(out=at(4)), G.GRACE_ERR_ALIAS),
    (dict(out=at(5)), G.GRACE_ERR_ALIAS),
    (dict(out=ctypes.c_void_p((6 << 24) + 4)), G.GRACE_ERR_ALIAS),      # inside residual, not residual itself
    (dict(R=0, x=None, out=None), G.GRACE_OK),
])
def test_linear_rejects(kw, status):
    assert linear(**kw) == status


def test_linear_binding_checks_every_tensor(monkeypatch):
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(G, "library", Library)
    x, w = torch.zeros(4, 64), torch.zeros(8, 64)
    for kw in (dict(w=torch.zeros(8, 63)), dict(bias=torch.zeros(4)), dict(residual=torch.zeros(8, 4)),
               dict(x_scale=torch.zeros(8)), dict(w_scale=torch.zeros(4)), dict(out=torch.zeros(4, 9)),
               dict(w=torch.zeros(64, 8).t()), dict(act="tanh")):
        with pytest.raises(ValueError):
            G.grace_linear(**{**dict(x=x, w=w), **kw})
    for kw in (dict(w=w.bfloat16()), dict(bias=torch.zeros(8).bfloat16()), dict(x=x.half()),
               dict(residual=torch.zeros(4, 8).double()), dict(x_scale=torch.zeros(4).bfloat16()),
               dict(out_dtype=torch.float8_e4m3fn)):
        with pytest.raises(TypeError):
            G.grace_linear(**{**dict(x=x, w=w), **kw})
    assert calls == []


def test_oracle_linear_by_hand():
    y = LO.linear([[1.0, 2.0]], [[3.0, -4.0]], bias=[1.0], act="relu", residual=[[0.5]])
    assert y == 0.5                                       # 3 - 8 + 1 < 0
    assert LO.linear([[1.0]], [[2.0]], x_scale=[3.0], w_scale=[5.0]) == 30.0
    assert abs(LO.linear([[1.0]], [[1.0]], act="gelu") - 0.8413447460685429) < 1e-15
    assert abs(LO.linear([[1.0]], [[1.0]], act="silu") - 0.7310585786300049) < 1e-15
