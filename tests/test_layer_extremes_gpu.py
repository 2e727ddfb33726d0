"""The position-wise entry points at ends of their ranges: more workgroups than one
launch takes, the tails of the activations, scales whose product leaves fp32."""
import math
import sys

import pytest
import torch

from paper_2608_00938_amd import grace as G

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _chunks(n, size=1 << 22):
    return [slice(i, min(n, i + size)) for i in range(0, n, size)]


@pytest.mark.parametrize("R,D", [((1 << 26) + 3, 4), ((1 << 21) + 3, 2056)])
def test_norm_of_very_many_rows(gpu, R, D):
    """Small integers: h is exact, and the tolerance that of test_norm_gpu.py twice over,
    for the fp32 arithmetic here, plus half a step of bf16."""
    _log(f"[extremes] norm R={R} D={D}")
    x = torch.randint(-8, 9, (R, D), device=gpu, dtype=torch.int8).to(BF16)
    w = torch.randint(1, 5, (D,), device=gpu).to(BF16)
    out = G.grace_rms_norm(x, w, 1e-6)
    for c in _chunks(R, (1 << 26) // D):
        h = x[c].float()
        want = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * w.float()
        assert ((out[c].float() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -17)).all(), c


@pytest.mark.parametrize("R,N,K", [(1, (1 << 27) + 5, 1), ((1 << 27) + 5, 8, 8), ((1 << 27) + 5, 1, 1)])
def test_linear_of_very_many_tiles(gpu, R, N, K):
    """Small integers: every sum is exact in fp32 and in bf16."""
    _log(f"[extremes] linear R={R} N={N} K={K}")
    x = torch.randint(-4, 5, (R, K), device=gpu, dtype=torch.int8).to(BF16)
    w = torch.randint(-4, 5, (N, K), device=gpu, dtype=torch.int8).to(BF16)
    out = G.grace_linear(x, w)
    if N > R:
        for c in _chunks(N):
            assert torch.equal(out[0, c], (x * w[c]).sum(1)), c
    else:
        for c in _chunks(R):
            want = sum(x[c, k:k + 1].float() * w[:, k].float() for k in range(K))
            assert torch.equal(out[c].float(), want), c


@pytest.mark.parametrize("R,V", [((1 << 26) + 5, 3), ((1 << 21) + 3, 4100)])
def test_sample_of_very_many_rows(gpu, R, V):
    _log(f"[extremes] sample R={R} V={V}")
    x = torch.randint(-40, 41, (R, V), device=gpu, dtype=torch.int8).to(BF16)
    cold = torch.zeros(1, device=gpu)
    tokens, scores = G.grace_sample(x, torch.zeros(R, device=gpu), 1, R, temperature=cold)
    place = torch.arange(V, device=gpu, dtype=torch.int32)
    for c in _chunks(R, (1 << 26) // V):
        top = x[c].amax(1, keepdim=True)
        first = torch.where(x[c] == top, place, V).amin(1)
        assert torch.equal(tokens[c], first.to(torch.int32)), c
        want = -(x[c].float() - top.float()).exp().sum(1).log()
        assert ((scores[c] - want).abs() <= 2.0 ** -16 * (1 + want.abs())).all(), c


def _tails():
    """y as bf16, where gelu(y) is a normal number."""
    y = torch.cat([torch.linspace(-12, 12, 3000), -torch.logspace(-30, 1, 600), torch.logspace(-30, 1, 600)])
    return y.to(BF16)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [16, 2048])
def test_gelu_keeps_relative_accuracy_in_its_tails(gpu, rows, out_dtype):
    """y (1 + erf) / 2 = y erfc(-y / sqrt 2) / 2.  The exponent y^2 / 2 (in powers of two at
    most 72 nepers here) is off by 5.5 * 2^-24 of itself: the rounded factor 1 / sqrt 2 (half) and
    product, both squared, log2(e) (half) and two products.  That is 2.4e-5 of the value; the
    rest, the tail's approximation among it, is below 2^-19 (32 steps).  Together less than
    2^-15, and the output's rounding."""
    y = _tails()
    x = torch.zeros(rows, 8, dtype=BF16)
    w = torch.zeros(8, 8, dtype=BF16)
    w[:, 0] = 1
    for i in range(0, len(y), rows):
        part = y[i:i + rows]
        x[:len(part), 0] = part
        got = G.grace_linear(x.to(gpu), w.to(gpu), act="gelu", out_dtype=out_dtype)[:len(part)].double().cpu()
        want = torch.tensor([v * math.erfc(-v / math.sqrt(2)) / 2 for v in part.tolist()], dtype=torch.float64)
        tol = want.abs() * (2.0 ** -15 + torch.finfo(out_dtype).eps / 2)
        assert ((got - want[:, None]).abs() <= tol[:, None]).all()


@pytest.mark.parametrize("R,N", [(3, 8), (100, 8), (100, 7)])
def test_scales_whose_product_leaves_fp32(gpu, R, N):
    """Powers of two, so that every order without an underflow is exact."""
    x = torch.full((R, 8), 2.0 ** 60, dtype=BF16, device=gpu)
    w = torch.full((N, 8), 2.0 ** 57, dtype=BF16, device=gpu)
    xs, ws = torch.full((R,), 2.0 ** -100, device=gpu), torch.full((N,), 2.0 ** -60, device=gpu)
    out = G.grace_linear(x, w, x_scale=xs, w_scale=ws, out_dtype=F32)
    assert (out == 2.0 ** -40).all()
