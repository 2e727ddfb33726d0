"""The position-wise entry points at ends of their ranges: more workgroups than one
launch takes."""
import sys

import numpy as np
import pytest
import torch

from paper_2608_00938_amd import grace as G

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


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
