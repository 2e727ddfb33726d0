"""grace_linear against its definition in fp64 on the same inputs.

Tolerances.  Products of bf16 or e4m3 values are exact in fp32; a sum of K of them
(of fp32 products, each rounded) in any order is within (K + 1) * 2^-23 of
A = sum |x w| even where every addition is off by a whole step.  Scales and bias
add three roundings of at most that kind, an activation's slope is at most 1.13
and its own arithmetic (exp, erf, division) is within 16 * 2^-23, the residual's
addition is one rounding more.  The output's rounding adds half a step: 2^-24
(fp32) or 2^-8 (bf16) of the value.

8-bit inputs with an output in bf16: each of the eight products of a group loses
less than 2^-13 of a power of two that is at most the largest product, so the
group is within 8 * 2^-13 = 2^-10 of its largest product and a sum within 2^-10 of A."""
import sys

import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO
from paper_2608_00938_amd import grace as G

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
STEP = 2.0 ** -23


def _log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _f64(t):
    return None if t is None else t.float().cpu().numpy().astype(np.float64)


def _inputs(dev, R, N, K, dtype, out_dtype, seed, bias=True, residual=True, scales=None):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
    x, w = draw(R, K), draw(N, K)
    s = dict(x=x.to(dtype), w=w.to(dtype))
    if dtype == E4M3 if scales is None else scales:
        s["x_scale"] = torch.exp(draw(R))
        s["w_scale"] = torch.exp(draw(N))
    if bias:
        s["bias"] = draw(N).to(out_dtype)
    if residual:
        s["residual"] = draw(R, N).to(out_dtype)
    return {k: v.to(dev) for k, v in s.items()}


def _check(got, s, act, out_dtype, rows=None):
    pick = (lambda t: t) if rows is None else (lambda t: None if t is None else t[rows])
    x, w = _f64(pick(s["x"])), _f64(s["w"])
    xs, ws = _f64(pick(s.get("x_scale"))), _f64(s.get("w_scale"))
    bias, res = _f64(s.get("bias")), _f64(pick(s.get("residual")))
    want = LO.linear(x, w, bias, act, res, xs, ws)
    pre = LO.linear(x, w, bias, "none", None, xs, ws)
    A = LO.linear(np.abs(x), np.abs(w), None, "none", None, xs, ws)
    size = A + (0 if bias is None else np.abs(bias)) + (0 if res is None else np.abs(res))
    tol = 1.13 * (x.shape[1] + 4) * STEP * A + 24 * STEP * (size + np.abs(pre)) + HALF[out_dtype] * np.abs(want)
    if s["x"].dtype == E4M3 and out_dtype == BF16:
        tol = tol + 1.13 * 2.0 ** -10 * A
    err = np.abs(_f64(pick(got)) - want)
    worst = float((err / tol).max())
    assert worst <= 1, worst


SIZES = [(1, 1, 1), (1, 512, 64), (5, 3, 7), (31, 33, 16), (33, 31, 129), (64, 64, 64), (65, 100, 63),
         (130, 129, 128), (17, 509, 1021), (257, 65, 200), (16, 1024, 512), (300, 520, 96), (1, 2048, 1024),
         (40, 40, 4096), (128, 256, 255), (2, 130, 2050)]


@pytest.mark.parametrize("R,N,K", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_linear_parity(gpu, R, N, K, dtype):
    for out_dtype in (F32, BF16):
        _log(f"[linear] R={R} N={N} K={K} {dtype} -> {out_dtype}")
        s = _inputs(gpu, R, N, K, dtype, out_dtype, 7 * R + N + K)
        got = G.grace_linear(**s, out_dtype=out_dtype)
        plain = {k: s[k] for k in ("x", "w")}
        bare = G.grace_linear(**plain, out_dtype=out_dtype)
        torch.cuda.synchronize()
        assert got.dtype == out_dtype
        _check(got, s, "none", out_dtype)
        _check(bare, plain, "none", out_dtype)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("R,N,K", [(50, 70, 48), (9, 256, 128), (200, 384, 256)])
def test_epilogues(gpu, act, dtype, R, N, K):
    for bias in (False, True):
        for residual in (False, True):
            for scales in (False, True):
                s = _inputs(gpu, R, N, K, dtype, BF16, 3, bias, residual, scales)
                got = G.grace_linear(**s, act=act, out_dtype=BF16)
                torch.cuda.synchronize()
                _check(got, s, act, BF16)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("R,N,K", [(33, 67, 40), (260, 512, 256), (1, 96, 64), (16, 64, 1024)])
def test_residual_in_place_and_nothing_else_written(gpu, dtype, R, N, K):
    """The output lies in the middle of a larger buffer whose other values stay."""
    s = _inputs(gpu, R, N, K, dtype, BF16, 5)
    want = G.grace_linear(**s, act="silu", out_dtype=BF16)
    pad = 64
    big = torch.full((R * N + 2 * pad,), 7.0, dtype=BF16, device=gpu)
    out = big[pad:pad + R * N].view(R, N)
    out.copy_(s["residual"])
    G.grace_linear(**{**s, "residual": out}, act="silu", out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert (big[:pad] == 7).all() and (big[-pad:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("R,N,K", [(70, 66, 128), (4, 128, 512)])
def test_tensors_off_16_bytes(gpu, dtype, R, N, K):
    """Contiguous views that start one element into their storage, in every place."""
    s = _inputs(gpu, R, N, K, dtype, F32, 9)
    want = _f64(G.grace_linear(**s, out_dtype=F32))

    def moved(t):
        big = torch.empty(t.numel() + 1, dtype=t.dtype, device=gpu)
        big[1:].copy_(t.reshape(-1))
        return big[1:].view(t.shape)

    for name in s:
        got = G.grace_linear(**{**s, name: moved(s[name])}, out_dtype=F32)
        torch.cuda.synchronize()
        _check(got, s, "none", F32)
    out = moved(torch.zeros(R, N, device=gpu))
    G.grace_linear(**s, out=out)
    torch.cuda.synchronize()
    _check(out, s, "none", F32)
    assert np.isfinite(want).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [64, 70, 1021])
def test_nan_and_inf_stay_in_their_row_and_column(gpu, dtype, K):
    """Also those that lie next to a row's end, which the last step of k reads over."""
    R, N = 40, 50
    s = _inputs(gpu, R, N, K, dtype, F32, 13, bias=False, residual=False)
    clean = G.grace_linear(**s)
    x, w = s["x"].clone(), s["w"].clone()
    x[7, 0] = float("nan")          # behind the end of row 6
    x[11, K - 1] = float("inf")
    w[3, 0] = float("inf")
    w[20, K - 1] = float("nan")
    got = G.grace_linear(x, w)
    torch.cuda.synchronize()
    rows = [r for r in range(R) if r not in (7, 11)]
    cols = [n for n in range(N) if n not in (3, 20)]
    assert torch.equal(got[rows][:, cols], clean[rows][:, cols])
    assert torch.isnan(got[7]).all() and torch.isnan(got[:, 20]).all()
    assert not torch.isfinite(got[11]).any() and not torch.isfinite(got[:, 3]).any()


def test_no_rows(gpu):
    assert G.grace_linear(torch.zeros(0, 64, device=gpu), torch.zeros(8, 64, device=gpu)).shape == (0, 8)


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("R,N,K", [(3, 512, 256), (300, 260, 128), (1024, 1024, 192)])
def test_other_stream_and_graph_replays(gpu, dtype, R, N, K):
    s = _inputs(gpu, R, N, K, dtype, BF16, 17)
    want = G.grace_linear(**s, act="gelu", out_dtype=BF16)
    out = torch.empty_like(want)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call = lambda: G.grace_linear(**s, act="gelu", out=out)  # noqa: E731
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    assert torch.equal(out, want)
    graph = G.capture(call, stream)
    for rep in range(3):
        out.fill_(3)
        G.grace_linear(**s, out_dtype=BF16)        # eager work between the replays
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        assert torch.equal(out, want), rep
    graph.destroy()


def test_more_than_2_31_outputs(gpu):
    """Offsets past 32 bits: the last rows of 2^31 + some outputs."""
    R, N, K = (1 << 20) + 40, 2048, 32
    s = _inputs(gpu, 40, N, K, BF16, BF16, 23, residual=False)
    x = torch.zeros((R, K), dtype=BF16, device=gpu)
    x[-40:] = s["x"]
    out = G.grace_linear(x, s["w"], bias=s["bias"])
    torch.cuda.synchronize()
    _check(out[-40:], s, "none", BF16)
    assert torch.equal(out[5], s["bias"])


def test_more_than_2_31_inputs(gpu):
    R, N, K = (1 << 15) + 3, 16, 1 << 16
    s = _inputs(gpu, 3, N, K, E4M3, F32, 29, bias=False, residual=False)
    x = torch.zeros((R, K), dtype=E4M3, device=gpu)
    x[-3:] = s["x"]
    out = G.grace_linear(x, s["w"], w_scale=s["w_scale"], out_dtype=F32)
    torch.cuda.synchronize()
    _check(out[-3:], {k: s[k] for k in ("x", "w", "w_scale")}, "none", F32)
    assert not out[:-3].any()


@pytest.mark.parametrize("R,N,K", [(33000, 520, 160), (20000, 1000, 328), (5000, 2056, 250), (70000, 136, 64),
                                   (33000, 515, 161), (1500, 1500, 1200), (66000, 260, 96), (300, 300, 4104)])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (E4M3, BF16), (E4M3, F32)])
def test_many_tiles(gpu, R, N, K, dtype, out_dtype):
    """Sizes that reach each of the tile sizes, with partial tiles in every direction;
    the first, last and some other rows."""
    s = _inputs(gpu, R, N, K, dtype, out_dtype, R + K)
    want_rows = np.unique(np.r_[0:70, R // 2:R // 2 + 70, R - 300:R])
    rows = torch.from_numpy(want_rows).to(gpu)
    got = G.grace_linear(**s, act="silu", out_dtype=out_dtype)
    torch.cuda.synchronize()
    _check(got, s, "silu", out_dtype, rows)
    assert torch.isfinite(got.float()).all()


@pytest.mark.parametrize("R,N,K", [(130, 200, 64), (300, 264, 104), (200, 4000, 100), (20, 30, 40)])
@pytest.mark.parametrize("x_size,w_size", [(2.0 ** -100, 1.0), (2.0 ** -118, 2.0 ** 20), (2.0 ** 100, 2.0 ** -60),
                                           (2.0 ** -60, 2.0 ** 60), (2.0 ** 120, 2.0 ** -100)])
def test_fp32_of_any_size(gpu, R, N, K, x_size, w_size):
    """Products next to either end of fp32's range are as exact as others."""
    s = _inputs(gpu, R, N, K, F32, F32, 31, bias=False, residual=False)
    s = {"x": s["x"] * x_size, "w": s["w"] * w_size}
    got = G.grace_linear(**s)
    torch.cuda.synchronize()
    _check(got, s, "none", F32)


@pytest.mark.parametrize("R,N,K", [(200, 300, 64), (300, 264, 33), (20, 30, 40)])
def test_fp32_infinities_and_largest_values(gpu, R, N, K):
    """As sums of products: an infinity times a number of either sign is one, times 0 NaN;
    the largest fp32 stays finite."""
    s = _inputs(gpu, R, N, K, F32, F32, 37, bias=True, residual=True)
    s["w"][3] = 0.0
    s["x"][5, 2] = float("inf")
    s["x"][9, K - 1] = torch.finfo(F32).max
    s["w"][:, K - 1] *= 2.0 ** -20
    s["w"][7, 0] = float("-inf")
    got = G.grace_linear(**s).cpu().numpy()
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want = (s["x"].cpu().double() @ s["w"].cpu().double().t() + s["bias"].cpu().double() +
                s["residual"].cpu().double()).numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want[5, 3])
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf].astype(np.float32)) and inf[5].sum() > N // 2
    fine = np.isfinite(want)
    assert np.isfinite(got[fine]).all()
    # the tolerance of the other tests, where neither row nor column holds an infinity
    with np.errstate(invalid="ignore"):
        A = np.abs(s["x"].cpu().double().numpy()) @ np.abs(s["w"].cpu().double().numpy()).T
        tol = 1.13 * (K + 28) * STEP * (A + 8)
    assert (np.abs(got[fine] - want[fine]) <= tol[fine]).all()


@pytest.mark.parametrize("K", [1, 31, 33, 65, 97, 130, 161, 193, 257, 383, 1021])
@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
def test_odd_rows_through_one_to_many_tiles(gpu, K, dtype):
    """Rows off 16 bytes in tiles of 128 bytes of k, several of which are under way at once;
    columns that end 1 to 7 into an eight, the residual updated in place."""
    for N in (509, 516, 519):
        out_dtype = F32 if dtype == F32 else BF16
        _log(f"[linear] odd rows K={K} N={N} {dtype}")
        s = _inputs(gpu, 1900, N, K, dtype, out_dtype, 31 * K + N)
        rows = torch.arange(0, 1900, 19, device=gpu)
        before = {**s, "residual": s["residual"].clone()}
        got = G.grace_linear(**s, act="relu", out=s["residual"])
        torch.cuda.synchronize()
        _check(got, before, "relu", out_dtype, rows)
