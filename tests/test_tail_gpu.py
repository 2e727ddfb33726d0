"""The decode loop with its tail (logits from the attention's output) and with
sampling, eager and as one replayed graph.

The tail's steps are checked one by one, each from the values that the one before
it left, with the tolerances of test_norm_gpu and test_linear_gpu; sampled tokens
against the oracle on the loop's own logits, exactly; trie nodes as the walk of
the sampled tokens."""
import sys

import numpy as np
import pytest
import torch

import test_linear_gpu as TL
import test_norm_gpu as TN
import test_sample_gpu as TS
from oracle import beam_oracle as BO
from oracle import gtm_oracle as GO
from oracle import layer_oracle as LO
from oracle import sample_oracle as SO
from paper_2608_00938_amd import decode as D
from paper_2608_00938_amd import grace as G
from paper_2608_00938_amd import workloads as W

pytestmark = pytest.mark.gpu


def _log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _tail(dev, width, Dm, F, V, seed, eight_bit, dt=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *shape: (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(dt).to(dev)  # noqa: E731
    one = lambda n: (1 + 0.1 * torch.randn(n, generator=g)).to(dt).to(dev)  # noqa: E731
    return D.DecodeTail(draw(Dm, width), draw(Dm, width), one(Dm), draw(F, Dm), draw(F), draw(Dm, F), one(Dm),
                        3 * draw(V, Dm), eight_bit=eight_bit)


def _loop(dev, widths, eight_bit=False, sampled=False, gtm=None, B=2, H=2, d=64, V=64, Dm=96, F=160, layers=2,
          seed=31):
    wl = W.custom(dtype="bf16", B=B, M=max(widths), H=H, d=d, steps=len(widths), L=24)
    inp = W.DecodeInputs(wl, seed, dev)
    ek, ev = inp.enc_kv
    steps = [[{tag: W.normal((B * M, H, d), seed + 100 * l, tag, t, wl, dev)
               for tag in ("q_cross", "q_self", "k_new", "v_new")} for t, M in enumerate(widths)]
             for l in range(layers)]
    hidden = [W.normal((B * M, Dm), seed + 7, "q_cross", t, wl, dev) for t, M in enumerate(widths)]
    masks = [torch.from_numpy(W.beam_mask(seed, t, B * M, V, keep=0.7).view(np.int32)).to(dev)
             for t, M in enumerate(widths)]
    sampling = None
    if sampled:
        g = torch.Generator().manual_seed(seed)
        rules = dict(temperature=torch.tensor([0.8, 1.1]), top_k=torch.tensor([20, 0], dtype=torch.int32),
                     top_p=torch.tensor([0.95, 0.9]), min_p=torch.tensor([0.0, 0.01]))
        sampling = D.Sampling([torch.rand(B * M, generator=g).to(dev) for M in widths],
                              **{k: v.to(dev) for k, v in rules.items()})
    tail = _tail(dev, H * d, Dm, F, V, seed, eight_bit)
    return D.DecodeLoop(B, widths, H, d, V, layers, ek, ev, inp.offsets_tensor(), steps, None, masks, gtm=gtm,
                        tail=tail, hidden=hidden, sampling=sampling)


@pytest.mark.parametrize("eight_bit", [False, True])
def test_tail_stage_by_stage(gpu, eight_bit):
    B, H, d, V, Dm, F, R = 3, 2, 64, 100, 96, 160, 45
    g = torch.Generator().manual_seed(5)
    draw = lambda *shape: torch.randn(shape, generator=g).bfloat16().to(gpu)  # noqa: E731
    tail = _tail(gpu, H * d, Dm, F, V, 3, eight_bit)
    hidden, xc, xs = draw(R, Dm), draw(R, H, d), draw(R, H, d)
    logits = torch.empty((R, V), dtype=torch.bfloat16, device=gpu)
    buf = tail.buffers(R + 3)
    tail.run(hidden, xc, xs, logits, buf)
    torch.cuda.synchronize()
    bf = torch.bfloat16
    out = {k: torch.empty_like(v[:R]) if v is not None else None for k, v in buf.items()}
    check = lambda got, act="none", **s: TL._check(got, {k: v for k, v in s.items() if v is not None}, act, bf)  # noqa: E731

    # the library's own steps once more, each output checked against the oracle
    h = G.grace_linear(xc.view(R, -1), tail.w_cross, residual=hidden)
    check(h, x=xc.view(R, -1), w=tail.w_cross, residual=hidden)
    attn = G.grace_linear(xs.view(R, -1), tail.w_self)
    check(attn, x=xs.view(R, -1), w=tail.w_self)
    h2 = torch.empty_like(h)

    def norm(x, weight, residual, total):
        got = G.grace_rms_norm(x, weight, tail.eps, residual=residual, sum_out=total, out=out["normed"],
                               out_scale=out["scale"])
        n, s = got if eight_bit else (got, None)
        hh, y = LO.rms_norm(_f64(x), _f64(weight), tail.eps, None if residual is None else _f64(residual))
        TN._check(n, s, y, n.dtype)
        return n.clone(), None if s is None else s.clone()

    n, s = norm(attn, tail.norm_ff, h, h2)
    up = G.grace_linear(n, tail.w_up, bias=tail.b_up, act=tail.act, x_scale=s, w_scale=tail.up_scale, out_dtype=bf)
    check(up, tail.act, x=n, w=tail.w_up, bias=tail.b_up, x_scale=s, w_scale=tail.up_scale)
    h3 = G.grace_linear(up, tail.w_down, residual=h2)
    check(h3, x=up, w=tail.w_down, residual=h2)
    n2, s2 = norm(h3, tail.norm_out, None, None)
    z = G.grace_linear(n2, tail.w_logits, x_scale=s2, w_scale=tail.logits_scale, out_dtype=bf)
    check(z, x=n2, w=tail.w_logits, x_scale=s2, w_scale=tail.logits_scale)
    torch.cuda.synchronize()
    # the tail, which updates its stream in place, ends at the same bits
    assert torch.equal(z, logits) and torch.equal(buf["h"][:R], h3) and torch.equal(buf["up"][:R], up)


def _outputs(loop):
    return loop.logits + loop.tokens + loop.scores + (loop.nodes[1:] if loop.gtm is not None else [])


@pytest.mark.parametrize("sampled", [False, True])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_loop_with_tail_replays(gpu, sampled, eight_bit):
    widths = (6, 6, 6) if sampled else (1, 8, 12)
    loop = _loop(gpu, widths, eight_bit, sampled)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        loop.run()
    stream.synchronize()
    want = [x.clone() for x in _outputs(loop)]
    assert all(torch.isfinite(x).all() for x in loop.logits)
    # the logits depend on the attention of this step
    assert not torch.equal(loop.logits[1][:1], loop.logits[2][:1])
    graph = loop.capture(stream)
    other = _loop(gpu, widths, eight_bit, sampled, seed=77)
    for rep in range(3):
        for x in _outputs(loop):
            x.fill_(-3)
        other.run()
        torch.cuda.synchronize()
        graph.launch(stream)
        stream.synchronize()
        for a, b in zip(_outputs(loop), want):
            assert torch.equal(a, b), rep
    graph.destroy()
    V, M = loop.V, widths[-1]
    for t, M in enumerate(widths):
        mask = BO.unpack_mask(loop.masks[t].cpu().numpy().view(np.uint32), V)
        prev = np.zeros(2 * M) if t == 0 else _f64(loop.scores[t - 1]).reshape(-1)
        if sampled:
            r = {k: v.cpu().numpy() for k, v in loop.sampling.rules.items()}
            tok, sc = SO.sample(_f64(loop.logits[t]), loop.sampling.uniform[t].cpu().numpy(), M, mask=mask,
                                T=r["temperature"], k=r["top_k"], p=r["top_p"], min_p=r["min_p"], prev=prev)
            assert np.array_equal(loop.tokens[t].cpu().numpy().reshape(-1), tok)
            assert np.abs(_f64(loop.scores[t]).reshape(-1) - sc).max() <= TS.SCORE
        else:
            cand = BO.candidate_scores(_f64(loop.logits[t]), prev, mask)
            got = cand.reshape(2, -1)[np.arange(2)[:, None], loop.parents[t].cpu().numpy().astype(np.int64) * V +
                                      loop.tokens[t].cpu().numpy()]
            best = -np.sort(-cand.reshape(2, -1), axis=1)[:, :loop.k_out[t]]
            assert np.abs(got - best)[np.isfinite(best)].max() <= 1e-4


def test_sampled_rows_follow_the_trie(gpu):
    """Sampling under the CD+GTM filter: a row's node is the walk of its tokens, and a
    row that the filter leaves nothing is dead from then on."""
    B, M, T = 2, 40, 4
    ix = W.gtm_index(41, 20000)
    us = W.gtm_users(41, B, L_max=16)
    loop = _loop(gpu, (M,) * T, sampled=True, gtm=(G.GtmIndex(ix, gpu), G.GtmUsers(us, gpu)), V=512)
    loop.run()
    torch.cuda.synchronize()
    assert int(loop.gtm_err.item()) == 0
    node = np.zeros(B * M, dtype=np.int32)
    own = np.tile(np.arange(M), B)
    alive = 0
    for t in range(T):
        tok = loop.tokens[t].cpu().numpy().reshape(-1)
        allowed = GO.gtm_mask(ix, us, node, B, M)
        assert np.array_equal(loop.masks[t].cpu().numpy().view(np.uint32), GO.pack_mask(allowed))
        dead = ~allowed.any(axis=1)
        assert np.array_equal(tok == -1, dead)
        live = np.flatnonzero(~dead)
        assert allowed[live, tok[live]].all()
        assert np.array_equal(np.isneginf(_f64(loop.scores[t]).reshape(-1)), dead)
        node = GO.trie_advance(ix, node, own, tok, B, M, M)
        assert np.array_equal(loop.nodes[t + 1].cpu().numpy(), node)
        alive = live.size
        _log(f"  step {t}: {alive} of {B * M} rows alive")
    assert alive > 0


def test_sampling_refuses_changing_widths(gpu):
    with pytest.raises(ValueError, match="widths"):
        _loop(gpu, (1, 8, 8), sampled=True)
    with pytest.raises(ValueError, match="logits"):
        loop = _loop(gpu, (2, 2))
        D.DecodeLoop(2, (2, 2), 2, 64, 65, 2, loop.enc_k, loop.enc_v, loop.enc_off, loop.inputs, None,
                     tail=loop.tail, hidden=loop.hidden)
