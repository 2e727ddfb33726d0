"""grace_sample against its definition in fp64.  Tokens are compared for equality.

Scores: prev + z - top - log(sum of exp) with every term below 2^7 here: four
roundings of at most 2^-18 (half a step of fp32 at 128), and the sum of exp, whose
terms are within 2^-20 of theirs (2 steps of exp and of its argument) and are added
in fp64 or, in fp32, in chains of at most 128 before a tree of 10: within
140 * 2^-24 < 2^-16.  Together below 2^-15."""
import sys

import numpy as np
import pytest
import torch

from oracle import beam_oracle as BO
from oracle import sample_oracle as SO
from paper_2608_00938_amd import grace as G

pytestmark = pytest.mark.gpu

SCORE = 2.0 ** -15


def _log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _pack(mask):
    """bool [R, V] -> int32 words."""
    R, V = mask.shape
    wide = np.zeros((R, (V + 31) // 32 * 32), dtype=bool)
    wide[:, :V] = mask
    words = np.packbits(wide, axis=1, bitorder="little").view(np.uint32)
    assert np.array_equal(BO.unpack_mask(words, V), mask)
    return torch.from_numpy(words.view(np.int32).copy())


def _logits(rng, R, V, dtype, kind):
    z = rng.standard_normal((R, V)) * 3
    if kind == "grid":
        z = np.round(z * 4) / 4
    elif kind == "equal":
        z = np.full((R, V), 1.5)
    elif kind == "peaked":
        z = z + 25 * (rng.random((R, V)) < 2.0 / V)
    elif kind == "wide":
        z = z * 15
    t = torch.from_numpy(z).to(torch.float32)
    return t.to(torch.bfloat16) if dtype == "bf16" else t


RULES = {
    "plain": {},
    "temperature": dict(T=[0.7, 1.3, 0.0]),
    "k": dict(k=[3, 50, 1]),
    "p": dict(p=[0.9, 0.5, 0.99]),
    "min_p": dict(min_p=[0.05, 0.3, 0.9]),
    "all": dict(T=[0.8, 1.0, 1.5], k=[40, 0, 7], p=[0.95, 0.8, 1.0], min_p=[0.0, 0.02, 0.01]),
}


def _run(dev, logits, u, B, M, mask=None, T=None, k=None, p=None, min_p=None, prev=None, **kw):
    f = lambda v, dt: None if v is None else torch.tensor(np.asarray(v), dtype=dt).to(dev)  # noqa: E731
    got = G.grace_sample(logits.to(dev), f(u, torch.float32), B, M, temperature=f(T, torch.float32),
                         top_k=f(k, torch.int32), top_p=f(p, torch.float32), min_p=f(min_p, torch.float32),
                         mask=None if mask is None else _pack(mask).to(dev), prev_scores=f(prev, torch.float32), **kw)
    torch.cuda.synchronize()
    return got


def _compare(dev, logits, u, B, M, **kw):
    f32 = lambda v: None if v is None else np.asarray(v, dtype=np.float32)  # noqa: E731
    tokens, scores = _run(dev, logits, u, B, M, **kw)
    z = logits.float().numpy()
    want, ws = SO.sample(z, u, M, mask=kw.get("mask"), T=f32(kw.get("T")), k=kw.get("k"), p=f32(kw.get("p")),
                         min_p=f32(kw.get("min_p")), prev=kw.get("prev"))
    tokens, scores = tokens.cpu().numpy(), scores.cpu().numpy().astype(np.float64)
    assert np.array_equal(tokens, want), np.flatnonzero(tokens != want)
    # a logit of finfo.min under one of finfo.max: its log-probability, -6.8e38, is past fp32
    ws = np.where(np.abs(ws) > np.finfo(np.float32).max, np.copysign(np.inf, ws), ws)
    fine = np.isfinite(ws)
    assert np.array_equal(np.isnan(ws), np.isnan(scores))
    assert np.array_equal(ws[~fine & ~np.isnan(ws)], scores[~fine & ~np.isnan(ws)])
    assert (np.abs(scores[fine] - ws[fine]) <= SCORE).all(), np.abs(scores[fine] - ws[fine]).max()
    return tokens


SIZES = [(3, 5, 1), (3, 4, 2), (3, 7, 7), (3, 9, 31), (3, 9, 32), (3, 8, 33), (3, 20, 64), (3, 6, 100),
         (3, 33, 257), (3, 40, 509), (3, 200, 512), (3, 21, 520), (3, 10, 1000), (3, 11, 1024), (3, 9, 2000),
         (3, 7, 2048), (3, 5, 4096), (3, 5, 4097), (3, 3, 4104), (3, 2, 10007), (3, 1, 32768), (3, 1, 50257),
         (3, 1, 128000)]


@pytest.mark.parametrize("B,M,V", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rules", RULES)
def test_sample_parity(gpu, B, M, V, dtype, rules):
    _log(f"[sample] B={B} M={M} V={V} {dtype} {rules}")
    rng = np.random.default_rng([V, len(rules), dtype == "f32"])
    R = B * M
    u = rng.random(R, dtype=np.float32)
    prev = (-20 * rng.random(R)).astype(np.float32)
    for masked in (False, True):
        mask = rng.random((R, V)) < 0.6 if masked else None
        _compare(gpu, _logits(rng, R, V, dtype, "normal"), u, B, M, mask=mask, prev=prev, **RULES[rules])


@pytest.mark.parametrize("kind", ["grid", "equal", "peaked", "wide"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rules", RULES)
@pytest.mark.parametrize("B,M,V", [(3, 30, 64), (3, 50, 512), (3, 9, 1500), (3, 3, 6000), (3, 1, 40000)])
def test_ties_and_distributions(gpu, kind, dtype, rules, B, M, V):
    rng = np.random.default_rng([V, 5])
    R = B * M
    u = rng.random(R, dtype=np.float32)
    mask = rng.random((R, V)) < 0.5
    logits = _logits(rng, R, V, dtype, kind)
    _compare(gpu, logits, u, B, M, **RULES[rules])
    _compare(gpu, logits, u, B, M, mask=mask, **RULES[rules])


@pytest.mark.parametrize("V", [5, 64, 509, 512, 3000, 9000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_uniform_at_its_ends(gpu, V, dtype):
    rng = np.random.default_rng(V)
    u = np.array([0.0, -0.0, 1 - 2.0 ** -24, 1.0, 7.0, -3.0, np.nan, np.inf, -np.inf, 2.0 ** -149, 0.5, 1e-7],
                 dtype=np.float32)
    logits = _logits(rng, 12, V, dtype, "normal")
    _compare(gpu, logits, u, 1, 12)
    _compare(gpu, logits, u, 12, 1, mask=rng.random((12, V)) < 0.4, p=[0.9] * 12, k=[20] * 12)


@pytest.mark.parametrize("V", [6, 512, 1000, 8192])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rules_out_of_range(gpu, V, dtype):
    rng = np.random.default_rng(V + 1)
    nan, inf = float("nan"), float("inf")
    T = [0.0, -1.0, nan, 1e-30, 1e30, inf, 1e-40, 1.0]
    k = [0, -5, 1, V, V + 1, 2 ** 31 - 1, -2 ** 31, 2]
    p = [0.0, -1.0, nan, 1.0, 2.0, inf, 1e-6, -inf]
    m = [0.0, -1.0, nan, 1.0, 2.0, inf, 1e-30, -inf]
    B, M = 8, 3
    u = rng.random(B * M, dtype=np.float32)
    logits = _logits(rng, B * M, V, dtype, "normal")
    for rules in (dict(T=T), dict(k=k), dict(p=p), dict(min_p=m), dict(T=T, k=k, p=p, min_p=m),
                  dict(T=[1.0] * B, k=k, p=p[::-1], min_p=m[3:] + m[:3])):
        _compare(gpu, logits, u, B, M, **rules)


@pytest.mark.parametrize("V", [3, 40, 512, 1111, 7000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rules", ["plain", "p", "all"])
def test_rows_with_few_or_no_candidates(gpu, V, dtype, rules):
    """Rows that the mask or -inf empties, rows of one candidate, masks over the best
    tokens, NaN and +inf logits."""
    rng = np.random.default_rng(V + 2)
    B, M = 3, 6
    R = B * M
    logits = _logits(rng, R, V, dtype, "normal")
    mask = rng.random((R, V)) < 0.7
    mask[0] = False
    mask[1] = False
    mask[1, V - 1] = True
    logits[2] = -float("inf")
    logits[3] = -float("inf")
    logits[3, V // 2] = -50.0
    mask[3, V // 2] = True
    logits[4, 0] = float("nan")
    logits[5] = float("nan")
    logits[6, V - 1] = float("inf")
    mask[6, V - 1] = True
    logits[7, [0, V - 1]] = float("inf")
    mask[7] = True
    logits[8, V - 1] = float("inf")
    mask[8, V - 1] = False                     # +inf in a masked place
    logits[9, V // 2] = float("nan")
    mask[9, V // 2] = False                    # NaN in a masked place
    logits[10] = torch.finfo(logits.dtype).min
    logits[11] = torch.finfo(logits.dtype).min
    logits[11, 1] = torch.finfo(logits.dtype).max
    mask[12] = logits[12].float().numpy() < 0  # the best tokens are filtered
    u = rng.random(R, dtype=np.float32)
    tokens = _compare(gpu, logits, u, B, M, mask=mask, **RULES[rules])
    assert (tokens[[0, 2, 5]] == -1).all() and tokens[1] == V - 1
    _compare(gpu, logits, u, B, M, **RULES[rules])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [512, 520, 3000])
def test_views_off_16_bytes_and_scores_in_place(gpu, dtype, V):
    rng = np.random.default_rng(77)
    B, M = 3, 15
    R = B * M
    logits = _logits(rng, R, V, dtype, "normal")
    u = rng.random(R, dtype=np.float32)
    rules = RULES["all"]
    mask = rng.random((R, V)) < 0.6
    prev = (-5 * rng.random(R)).astype(np.float32)
    want = _run(gpu, logits, u, B, M, mask=mask, prev=prev, **rules)

    def moved(t):
        big = torch.empty(t.numel() + 1, dtype=t.dtype, device=gpu)
        big[1:].copy_(t.reshape(-1))
        return big[1:].view(t.shape)

    f = lambda v, dt: moved(torch.tensor(v, dtype=dt).to(gpu))  # noqa: E731
    scores = f(prev, torch.float32)
    guard = torch.full((R + 2,), -9, dtype=torch.int32, device=gpu)
    tokens, scores = G.grace_sample(
        moved(logits.to(gpu)), f(u, torch.float32), B, M, temperature=f(rules["T"], torch.float32),
        top_k=f(rules["k"], torch.int32), top_p=f(rules["p"], torch.float32),
        min_p=f(rules["min_p"], torch.float32), mask=moved(_pack(mask).to(gpu)), prev_scores=scores,
        scores=scores, tokens=guard[1:-1])
    torch.cuda.synchronize()
    assert torch.equal(tokens, want[0]) and int(guard[0]) == -9 and int(guard[-1]) == -9
    assert float((scores - want[1]).abs().max()) <= 2 * SCORE


def test_no_rows(gpu):
    t, s = G.grace_sample(torch.zeros(0, 64, device=gpu), torch.zeros(0, device=gpu), 0, 5)
    assert t.shape == (0,) and s.shape == (0,)


@pytest.mark.parametrize("B,M,V", [(4, 300, 512), (8, 1, 60000), (4, 16, 5000)])
def test_other_stream_and_graph_replays(gpu, B, M, V):
    rng = np.random.default_rng(3)
    R = B * M
    logits = _logits(rng, R, V, "bf16", "normal").to(gpu)
    u = torch.from_numpy(rng.random(R, dtype=np.float32)).to(gpu)
    T = torch.full((B,), 0.9, device=gpu)
    p = torch.full((B,), 0.95, device=gpu)
    k = torch.full((B,), 60, dtype=torch.int32, device=gpu)
    want, ws = G.grace_sample(logits, u, B, M, temperature=T, top_k=k, top_p=p)
    tokens, scores = torch.empty_like(want), torch.empty_like(ws)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call = lambda: G.grace_sample(logits, u, B, M, temperature=T, top_k=k, top_p=p, tokens=tokens,  # noqa: E731
                                  scores=scores)
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    assert torch.equal(tokens, want) and torch.equal(scores, ws)
    graph = G.capture(call, stream)
    for rep in range(3):
        tokens.fill_(-5)
        scores.fill_(7)
        G.grace_sample(logits, u, B, M)            # eager work between the replays
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        assert torch.equal(tokens, want) and torch.equal(scores, ws), rep
    graph.destroy()


@pytest.mark.parametrize("V", [512, 65536])
def test_more_than_2_31_logits(gpu, V):
    """Offsets past 32 bits: the last rows of 2^31 + some logits."""
    R = (1 << 31) // V + 6
    tail = _logits(np.random.default_rng(9), 6, V, "bf16", "normal")
    u = torch.rand(R, generator=torch.Generator().manual_seed(1))
    logits = torch.zeros((R, V), dtype=torch.bfloat16, device=gpu)
    logits[-6:] = tail.to(gpu)
    mask = torch.full((R, V // 32), -1, dtype=torch.int32, device=gpu)
    tokens, scores = G.grace_sample(logits, u.to(gpu), 1, R, mask=mask)
    torch.cuda.synchronize()
    want, ws = SO.sample(tail.float().numpy(), u[-6:].numpy(), 6)
    assert np.array_equal(tokens[-6:].cpu().numpy(), want)
    assert np.abs(scores[-6:].cpu().numpy() - ws).max() <= SCORE
    assert torch.equal(tokens[:100].cpu(), (u[:100].double() * V).floor().int())
