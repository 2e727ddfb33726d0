"""A fixed-length decode loop over the library's calls, capturable as one graph.

Per step t (beam width M_t per request) and decoder layer l:
cross-attention of the beams over the request's encoder K/V (Sec. 5.1), then
the fused paged append + self-attention (Sec. 5.2, Sec. 5.3) whose parents are
the previous step's top-k output.  After the layers, the constraint filter
(CD + GTM, Sec. 4, Sec. 5.4) of the beams' trie nodes, the beam score update (Sec. 3.1)
and top-k with k = M_{t+1} (Sec. 3.3) produce the next step's parents, prefix
scores and trie nodes on the device, so the whole loop runs without a host
round trip and is recorded as one graph (Sec. 5).

Inputs the model would compute (per-step queries, the current token's k/v and
the next-token logits, and the constraint filter's mask) are given as tensors;
with a :class:`DecodeTail` the logits come from the last layer's attention
instead: its projections onto the residual stream, the feed-forward, the norms
and the output matrix.  With :class:`Sampling` every row draws its next token
where the beam step searches.  This module only orchestrates: every buffer is
allocated at construction and ``run`` only enqueues library calls.
"""
from __future__ import annotations

import math

import torch

from . import grace as G


class DecodeTail:
    """The position-wise end of a decode step, from the last layer's attention to the logits:

        h = hidden + x_cross w_cross^T,   h += x_self w_self^T
        h += act(norm(h) w_up^T + b_up) w_down^T
        logits = norm(h) w_logits^T

    Weights are [out, in] of one dtype (fp32 or bf16), norm weights [D], b_up [F].
    ``eight_bit``: the norms' outputs, w_up and w_logits are e4m3 with a scale per
    row, the weights quantised here once."""

    def __init__(self, w_cross, w_self, norm_ff, w_up, b_up, w_down, norm_out, w_logits,
                 act: str = "silu", eps: float = 1e-6, eight_bit: bool = False):
        self.w_cross, self.w_self, self.w_down = w_cross, w_self, w_down
        self.norm_ff, self.norm_out, self.b_up = norm_ff, norm_out, b_up
        self.act, self.eps, self.eight_bit = act, eps, eight_bit
        quantise = self._quantise if eight_bit else (lambda w: (w, None))
        self.w_up, self.up_scale = quantise(w_up)
        self.w_logits, self.logits_scale = quantise(w_logits)
        self.D, self.F, self.V = w_cross.shape[0], w_up.shape[0], w_logits.shape[0]

    @staticmethod
    def _quantise(w):
        scale = w.float().abs().amax(1).clamp_min(2.0 ** -96) / 448
        return (w.float() / scale[:, None]).to(torch.float8_e4m3fn), scale

    def buffers(self, rows: int) -> dict:
        """What ``run`` writes on the way, for up to ``rows`` rows."""
        dt, dev = self.w_cross.dtype, self.w_cross.device
        make = lambda n, t=dt: torch.empty((rows, n), dtype=t, device=dev)  # noqa: E731
        normed = make(self.D, torch.float8_e4m3fn if self.eight_bit else dt)
        scale = torch.empty((rows,), dtype=torch.float32, device=dev) if self.eight_bit else None
        return dict(h=make(self.D), attn=make(self.D), normed=normed, scale=scale, up=make(self.F))

    def run(self, hidden, x_cross, x_self, logits, buffers):
        """Enqueue the tail of R rows: hidden [R, D], x_cross and x_self [R, H, d], logits [R, V]."""
        R = hidden.shape[0]
        b = {k: v if v is None else v[:R] for k, v in buffers.items()}
        G.grace_linear(x_cross.view(R, -1), self.w_cross, residual=hidden, out=b["h"])
        G.grace_linear(x_self.view(R, -1), self.w_self, out=b["attn"])
        G.grace_rms_norm(b["attn"], self.norm_ff, self.eps, residual=b["h"], sum_out=b["h"],
                         out=b["normed"], out_scale=b["scale"])
        G.grace_linear(b["normed"], self.w_up, bias=self.b_up, act=self.act, x_scale=b["scale"],
                       w_scale=self.up_scale, out=b["up"])
        G.grace_linear(b["up"], self.w_down, residual=b["h"], out=b["h"])
        G.grace_rms_norm(b["h"], self.norm_out, self.eps, out=b["normed"], out_scale=b["scale"])
        G.grace_linear(b["normed"], self.w_logits, x_scale=b["scale"], w_scale=self.logits_scale,
                       out=logits)


class Sampling:
    """Rules of a sampled decode, device tensors: uniform[t] fp32 [B*M], the random numbers
    of step t; temperature, top_p, min_p fp32 [B] and top_k int32 [B], or None."""

    def __init__(self, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
        self.uniform = uniform
        self.rules = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


class DecodeLoop:
    def __init__(self, B: int, widths, H: int, d: int, V: int, layers: int, enc_k, enc_v,
                 enc_off, step_inputs, logits, masks=None, k_final: int | None = None,
                 scale: float | None = None, gtm=None, tail: DecodeTail | None = None, hidden=None,
                 sampling: Sampling | None = None):
        """widths: beams per request at each step (M_0, ..., M_{T-1}).
        step_inputs[l][t]: dict(q_cross, q_self, k_new, v_new), each [B*M_t, H, d].
        logits[t]: [B*M_t, V]; masks[t]: packed filter words (int32 [B*M_t, ceil(V/32)]) or None.
        gtm: (GtmIndex, GtmUsers) to compute the filter of every step from the
        beams' trie nodes instead (masks is then ignored); beams start at the root.
        The top-k of step t keeps M_{t+1} beams; the last keeps k_final (default M_{T-1}).
        tail: computes the logits of every step from the last layer's attention and
        hidden[t] [B*M_t, D], the residual stream ahead of it (logits is then ignored).
        sampling: every row draws its next token instead; all widths are then one M,
        and a row stays its own parent."""
        self.B, self.widths, self.H, self.d, self.V, self.layers = B, tuple(widths), H, d, V, layers
        self.T = len(self.widths)
        self.enc_k, self.enc_v, self.enc_off = enc_k, enc_v, enc_off
        self.inputs, self.logits = step_inputs, logits
        self.masks = masks if masks is not None else [None] * self.T
        self.scale = 1.0 / math.sqrt(d) if scale is None else scale
        dev, dt = enc_k.device, enc_k.dtype
        Mmax = max(self.widths)
        self.caches = [G.KVCache(B, Mmax, H, d, self.T, dt, dev) for _ in range(layers)]
        self.k_out = [self.widths[t + 1] for t in range(self.T - 1)] + [k_final or self.widths[-1]]
        self.x_cross = [[torch.empty((B * M, H, d), dtype=dt, device=dev) for M in self.widths]
                        for _ in range(layers)]
        self.x_self = [[torch.empty((B * M, H, d), dtype=dt, device=dev) for M in self.widths]
                       for _ in range(layers)]
        self.prev0 = torch.zeros((B * self.widths[0],), dtype=torch.float32, device=dev)
        self.parents = [torch.empty((B, k), dtype=torch.int32, device=dev) for k in self.k_out]
        self.tokens = [torch.empty((B, k), dtype=torch.int32, device=dev) for k in self.k_out]
        self.scores = [torch.empty((B, k), dtype=torch.float32, device=dev) for k in self.k_out]
        ws = max(G.grace_beam_step_workspace_bytes(B, M, V) for M in self.widths)
        self.workspace = torch.empty((max(ws, 8),), dtype=torch.uint8, device=dev)
        self.tail, self.hidden = tail, hidden
        if tail is not None:
            if tail.V != V:
                raise ValueError(f"the tail has {tail.V} logits, not {V}")
            self.logits = [torch.empty((B * M, V), dtype=dt, device=dev) for M in self.widths]
            self.tail_buffers = tail.buffers(B * Mmax)
        self.sampling = sampling
        if sampling is not None:
            if set(self.widths) != {Mmax} or set(self.k_out) != {Mmax}:
                raise ValueError("sampled rows keep their places: all widths must be equal")
            own = torch.arange(Mmax, dtype=torch.int32, device=dev).repeat(B, 1)
            self.parents = [own] * self.T
        self.gtm = gtm
        if gtm is not None:
            W = (V + 31) // 32
            self.masks = [torch.empty((B * M, W), dtype=torch.int32, device=dev) for M in self.widths]
            self.nodes = [torch.zeros((B * self.widths[0],), dtype=torch.int32, device=dev)] + \
                [torch.empty((B * k,), dtype=torch.int32, device=dev) for k in self.k_out]
            self.gtm_err = torch.zeros(1, dtype=torch.int32, device=dev)

    def run(self):
        """Enqueue the whole loop on the current stream."""
        B = self.B
        for t, M in enumerate(self.widths):
            M_prev = self.widths[t - 1] if t > 0 else 1
            par = self.parents[t - 1].view(-1) if t > 0 else None
            for l in range(self.layers):
                x = self.inputs[l][t]
                G.grace_cross_attn(x["q_cross"], self.enc_k, self.enc_v, self.enc_off, M,
                                   self.scale, out=self.x_cross[l][t])
                self.caches[l].append_attend_dyn(t, x["q_self"], x["k_new"], x["v_new"], par,
                                                 M_prev, M, self.scale, out=self.x_self[l][t])
            prev = self.prev0 if t == 0 else self.scores[t - 1].view(-1)
            if self.gtm is not None:
                index, users = self.gtm
                G.grace_gtm_mask(index, users, self.nodes[t], B, M, mask=self.masks[t],
                                 err_flag=self.gtm_err)
            if self.tail is not None:
                self.tail.run(self.hidden[t], self.x_cross[-1][t], self.x_self[-1][t], self.logits[t],
                              self.tail_buffers)
            if self.sampling is not None:
                G.grace_sample(self.logits[t], self.sampling.uniform[t], B, M, mask=self.masks[t],
                               prev_scores=prev, tokens=self.tokens[t].view(-1),
                               scores=self.scores[t].view(-1), **self.sampling.rules)
            else:
                # score update + top-k in one call: no [B*M, V] candidate array
                G.grace_beam_step(self.logits[t], prev, B, M, self.k_out[t], mask=self.masks[t],
                                  parents=self.parents[t], tokens=self.tokens[t],
                                  scores=self.scores[t], workspace=self.workspace)
            if self.gtm is not None:
                G.grace_trie_advance(self.gtm[0], self.nodes[t], self.parents[t].view(-1),
                                     self.tokens[t].view(-1), B, M, self.k_out[t],
                                     node_next=self.nodes[t + 1], err_flag=self.gtm_err)

    def capture(self, stream) -> "G.Graph":
        """Record run() on ``stream`` (not the null stream) as one graph."""
        return G.capture(self.run, stream)
