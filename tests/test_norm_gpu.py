"""grace_rms_norm against its definition in fp64 on the same inputs.

Tolerances.  h is one fp32 addition of exact inputs (2^-24 relative); the mean of
squares is a sum of positive terms, at most 33 in a row in one lane and 10 to 26
more in a tree, so its relative error is below 64 * 2^-24 = 2^-18 and that of its
root half of it; two products follow.  Each output element is therefore within
2^-18 relative of the definition before its own rounding, which adds half a step:
2^-24 (fp32), 2^-8 (bf16), 2^-4 (e4m3; half of 2^-9 of the scale below 2^-6)."""
import sys

import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO
from paper_2608_00938_amd import grace as G

pytestmark = pytest.mark.gpu

EPS = 1e-6
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}
COMPUTE = 2.0 ** -18


def _log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _inputs(dev, R, D, dtype, seed, residual=True):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
    x = (draw(R, D) * torch.exp(draw(R, 1))).to(dtype).to(dev)
    res = (draw(R, D) * 3).to(dtype).to(dev) if residual else None
    return x, (1 + 0.2 * draw(D)).to(dtype).to(dev), res


def _check(out, scale, y, out_dtype):
    if out_dtype != torch.float8_e4m3fn:
        err = np.abs(_f64(out) - y)
        assert (err <= (HALF[out_dtype] + COMPUTE) * np.abs(y)).all(), (err / np.abs(y)).max()
        return
    s = _f64(scale)
    want = np.maximum(np.abs(y).max(axis=1), LO.TINY) / LO.E4M3_MAX
    assert (np.abs(s - want) <= 2 * COMPUTE * want).all()
    got = _f64(out) * s[:, None]
    tol = np.maximum(HALF[out_dtype] * np.abs(y), 2.0 ** -10 * want[:, None]) + 4 * COMPUTE * np.abs(y)
    assert (np.abs(got - y) <= tol).all()


# rows of one element, around a wave's and a workgroup's capacity, odd and even,
# up to the longest
@pytest.mark.parametrize("D", [1, 7, 8, 64, 100, 513, 1021, 1024, 2048, 2049, 2056, 4096, 8192, 8193,
                               8200, 32760, 32768])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16, torch.float8_e4m3fn])
def test_norm_parity(gpu, D, dtype, out_dtype):
    R = 5 if D > 4096 else 67
    x, w, res = _inputs(gpu, R, D, dtype, 11 + D)
    _log(f"[norm] R={R} D={D} {dtype} -> {out_dtype}")
    for residual in (None, res):
        h, y = LO.rms_norm(_f64(x), _f64(w), EPS, None if residual is None else _f64(residual))
        s = torch.full_like(x, 7.0)
        got = G.grace_rms_norm(x, w, EPS, residual=residual, sum_out=s, out_dtype=out_dtype)
        torch.cuda.synchronize()
        out, scale = got if out_dtype == torch.float8_e4m3fn else (got, None)
        assert out.dtype == out_dtype
        _check(out, scale, y, out_dtype)
        assert (np.abs(_f64(s) - h) <= (HALF[dtype] + 2.0 ** -24) * np.abs(h)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("which", ["x", "residual"])
@pytest.mark.parametrize("D", [1000, 1021, 4096, 20000])
def test_sum_in_place(gpu, dtype, which, D):
    x, w, res = _inputs(gpu, 9, D, dtype, 3)
    want_sum = torch.empty_like(x)
    want = G.grace_rms_norm(x, w, EPS, residual=res, sum_out=want_sum)
    a, b = x.clone(), res.clone()
    got = G.grace_rms_norm(a, w, EPS, residual=b, sum_out=a if which == "x" else b)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert torch.equal(a if which == "x" else b, want_sum)
    assert torch.equal(b if which == "x" else a, res if which == "x" else x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_off_16_bytes(gpu, dtype):
    """Contiguous views that start one element into their storage, in every place."""
    R, D = 6, 1024
    x, w, res = _inputs(gpu, R, D, dtype, 5)

    def moved(t):
        big = torch.empty(t.numel() + 1, dtype=t.dtype, device=gpu)
        big[1:].copy_(t.reshape(-1))
        return big[1:].view(t.shape)

    want = G.grace_rms_norm(x, w, EPS, residual=res)
    for a, b, c in ((moved(x), w, res), (x, moved(w), res), (x, w, moved(res))):
        got = G.grace_rms_norm(a, b, EPS, residual=c)
        torch.cuda.synchronize()
        assert (np.abs(_f64(got) - _f64(want)) <= (2 * HALF[dtype] + COMPUTE) * np.abs(_f64(want))).all()
    guard = torch.full((R * D + 1,), 7.0, dtype=dtype, device=gpu)
    G.grace_rms_norm(x, w, EPS, residual=res, out=guard[1:].view(R, D))
    torch.cuda.synchronize()
    assert float(guard[0]) == 7.0


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_zero_nan_and_inf_rows_stay_alone(gpu, out_dtype):
    x, w, _ = _inputs(gpu, 8, 640, torch.bfloat16, 9)
    clean = G.grace_rms_norm(x, w, EPS, out_dtype=out_dtype)
    y = x.clone()
    y[1] = 0
    y[3, 5] = float("nan")
    y[5, 639] = float("inf")
    got = G.grace_rms_norm(y, w, EPS, out_dtype=out_dtype)
    torch.cuda.synchronize()
    keep = [0, 2, 4, 6, 7]
    if out_dtype == torch.float8_e4m3fn:
        assert torch.equal(got[0].view(torch.uint8)[keep], clean[0].view(torch.uint8)[keep])
        assert torch.equal(got[1][keep], clean[1][keep])
        assert float(got[1][1]) == np.float32(LO.TINY / LO.E4M3_MAX) and not got[0][1].float().any()
        assert torch.isnan(got[1][3])
    else:
        assert torch.equal(got[keep], clean[keep])
        assert not got[1].any() and torch.isnan(got[3]).all()


def test_no_rows(gpu):
    x, w, _ = _inputs(gpu, 4, 64, torch.float32, 1)
    assert G.grace_rms_norm(x[:0], w).shape == (0, 64)


def test_other_stream_and_graph_replays(gpu):
    R, D = 300, 2048
    x, w, res = _inputs(gpu, R, D, torch.bfloat16, 21)
    want_sum = torch.empty_like(x)
    want, want_scale = G.grace_rms_norm(x, w, EPS, residual=res, sum_out=want_sum,
                                        out_dtype=torch.float8_e4m3fn)
    out, scale = torch.empty_like(want), torch.empty_like(want_scale)
    s = torch.empty_like(x)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call = lambda: G.grace_rms_norm(x, w, EPS, residual=res, sum_out=s, out=out, out_scale=scale)  # noqa: E731
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    assert torch.equal(out.view(torch.uint8), want.view(torch.uint8)) and torch.equal(s, want_sum)
    graph = G.capture(call, stream)
    for rep in range(3):
        out.view(torch.uint8).fill_(1)
        scale.fill_(-1)
        s.fill_(5)
        G.grace_rms_norm(x, w, EPS)                 # eager work between the replays
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        assert torch.equal(out.view(torch.uint8), want.view(torch.uint8)), rep
        assert torch.equal(scale, want_scale) and torch.equal(s, want_sum), rep
    graph.destroy()


def test_more_than_2_31_elements(gpu):
    """Offsets past 32 bits: the last rows of 2^31 + some elements."""
    R, D = (1 << 20) + 40, 2048
    x = torch.zeros((R, D), dtype=torch.bfloat16, device=gpu)
    tail, w, _ = _inputs(gpu, 40, D, torch.bfloat16, 2)
    x[-40:] = tail
    out = G.grace_rms_norm(x, w, EPS)
    want = G.grace_rms_norm(tail, w, EPS)
    torch.cuda.synchronize()
    assert torch.equal(out[-40:], want)
    assert not out[:64].any()
