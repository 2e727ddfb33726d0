"""Host checks of the position-wise entry points: bad arguments are refused
before any launch (no GPU: every call here returns from those checks)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO
from oracle import sample_oracle as SO
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


def sample(**kw):
    a = dict(z=at(1), u=at(2), prev=at(3), mask=at(4), T=at(5), k=at(6), p=at(7), m=at(8), B=2, M=4, V=64,
             dtype=G.GRACE_BF16, tok=at(10), sc=at(11))
    a.update(kw)
    return G.library().grace_sample(a["z"], a["u"], a["prev"], a["mask"], a["T"], a["k"], a["p"], a["m"],
                                    a["B"], a["M"], a["V"], a["dtype"], a["tok"], a["sc"], None)


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), G.GRACE_ERR_UNSUPPORTED), (dict(B=-1), G.GRACE_ERR_SHAPE), (dict(M=-1), G.GRACE_ERR_SHAPE),
    (dict(V=0), G.GRACE_ERR_SHAPE), (dict(V=(1 << 24) + 1), G.GRACE_ERR_SHAPE),
    (dict(B=1 << 16, M=1 << 15), G.GRACE_ERR_SHAPE), (dict(B=1 << 10, M=1 << 10, V=1 << 20), G.GRACE_ERR_SHAPE),
    (dict(z=None), G.GRACE_ERR_NULL), (dict(u=None), G.GRACE_ERR_NULL), (dict(tok=None), G.GRACE_ERR_NULL),
    (dict(sc=None), G.GRACE_ERR_NULL),
    (dict(tok=at(1)), G.GRACE_ERR_ALIAS), (dict(tok=at(2)), G.GRACE_ERR_ALIAS),
    (dict(tok=at(3)), G.GRACE_ERR_ALIAS), (dict(sc=at(4)), G.GRACE_ERR_ALIAS),
    (dict(sc=at(5)), G.GRACE_ERR_ALIAS), (dict(sc=at(6)), G.GRACE_ERR_ALIAS),
    (dict(sc=at(7)), G.GRACE_ERR_ALIAS), (dict(tok=at(8)), G.GRACE_ERR_ALIAS),
    (dict(sc=at(10)), G.GRACE_ERR_ALIAS),
    (dict(sc=ctypes.c_void_p((3 << 24) + 4)), G.GRACE_ERR_ALIAS),       # inside prev, not prev itself
    (dict(B=0, z=None), G.GRACE_OK), (dict(M=0, tok=None), G.GRACE_OK),
])
def test_sample_rejects(kw, status):
    assert sample(**kw) == status


def test_sample_binding_checks_every_tensor(monkeypatch):
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(G, "library", Library)
    i32 = torch.int32
    z, u = torch.zeros(6, 40), torch.zeros(6)
    for kw in (dict(B=3), dict(uniform=torch.zeros(5)), dict(prev_scores=torch.zeros(2)),
               dict(mask=torch.zeros(6, 1, dtype=i32)), dict(temperature=torch.zeros(6)),
               dict(top_k=torch.zeros(6, dtype=i32)), dict(top_p=torch.zeros(3)), dict(min_p=torch.zeros(1)),
               dict(tokens=torch.zeros(7, dtype=i32)), dict(scores=torch.zeros(2, 3)),
               dict(logits=torch.zeros(40, 6).t())):
        with pytest.raises(ValueError):
            G.grace_sample(**{**dict(logits=z, uniform=u, B=2, M=3), **kw})
    for kw in (dict(logits=z.half()), dict(uniform=u.double()), dict(top_k=torch.zeros(2)),
               dict(mask=torch.zeros(6, 2, dtype=torch.int64)), dict(tokens=torch.zeros(6, dtype=torch.int64)),
               dict(temperature=torch.zeros(2).bfloat16())):
        with pytest.raises(TypeError):
            G.grace_sample(**{**dict(logits=z, uniform=u, B=2, M=3), **kw})
    assert calls == []


def test_oracle_sampling_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    pick = lambda u, **kw: SO.sample_row(z, u, **kw)  # noqa: E731
    assert [pick(u) for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert list(SO.kept_tokens(z, k=2)[0]) == [1, 3]
    assert [pick(u, k=2) for u in (0.0, 0.57, 0.58)] == [1, 1, 3]          # 4/7
    assert list(SO.kept_tokens(z, p=0.65)[0]) == [1, 3] and list(SO.kept_tokens(z, p=0.75)[0]) == [1, 3, 2]
    assert list(SO.kept_tokens(z, k=3, p=0.75)[0]) == [1, 3]               # 0.7 of 0.9 reaches 0.675
    assert list(SO.kept_tokens(z, min_p=0.45)[0]) == [1, 3, 2]
    assert list(SO.kept_tokens(z, T=0.0)[0]) == [1] and list(SO.kept_tokens(z, p=0.0)[0]) == [1]
    assert list(SO.kept_tokens(z, allowed=[1, 0, 1, 0])[0]) == [2, 0]
    assert pick(0.5, allowed=[0, 0, 0, 0]) == -1
    w = SO.kept_tokens(z, T=0.5)[1]                                        # squares of the odds
    assert np.allclose(w, np.array([1, 9 / 16, 1 / 4, 1 / 16]))
    # ties: the lower token first, and equal logits weigh the same
    assert list(SO.kept_tokens(np.zeros(4), k=3)[0]) == [0, 1, 2]
    assert list(SO.kept_tokens(np.zeros(4), p=0.5)[0]) == [0, 1]
