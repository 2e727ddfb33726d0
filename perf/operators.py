"""The position-wise operators of a decode step as calls to be measured: the residual
stream's norm, the matrix product with its epilogue, and sampling.

A case is a dict of plain values; ``op`` names the operator:

  norm     grace_rms_norm  h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight
  linear   grace_linear    act(scales * x w^T + bias) + residual
  sample   grace_sample    a token per row, by temperature, top-k, top-p and min-p

``run`` computes them with elementary torch operations, or, where ``own`` is true,
with the library's entry points.
"""
import math

import torch

own = False

EPS = 1e-6
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
TINY = 2.0 ** -96          # least row maximum that a scale of the 8-bit output is made from
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}


def listed():
    norm = dict(op="norm", residual=True)
    linear = dict(op="linear", bias=False, act="none", residual=False)
    sample = dict(op="sample", mask=True, top_k=0, top_p=1.0, min_p=0.0, greedy=0.0)
    return [
        # first position: one beam for each of 64 requests, 16 x 64 heads; latency
        dict(norm, name="norm_r64_d1024", R=64, D=1024, dtype="bf16", out="bf16"),
        # 16 x 1024 beams, 16 x 128 heads, into an 8-bit matrix product
        dict(norm, name="norm_e4m3_r16384_d2048", R=16384, D=2048, dtype="bf16", out="e4m3"),
        # 64 x 4096 beams, 16 x 64 heads: the largest decode step
        dict(norm, name="norm_r262144_d1024", R=262144, D=1024, dtype="bf16", out="bf16"),
        # fp32 and odd sizes: rows that are no multiple of 16 bytes, no residual
        dict(norm, name="norm_f32_r3001_d1021", R=3001, D=1021, dtype="f32", out="f32", residual=False),
        # first feed-forward product of 16 beams: the weights' reading counts
        dict(linear, name="linear_r16_k1024_n4096", R=16, K=1024, N=4096, dtype="bf16", out="bf16",
             bias=True, act="gelu"),
        # output projection of 16 x 1024 beams with 16 x 128 heads, onto the residual stream
        dict(linear, name="linear_r16384_k2048_n2048", R=16384, K=2048, N=2048, dtype="bf16",
             out="bf16", residual=True),
        # first feed-forward product of 64 x 4096 beams in 8 bits: the largest
        dict(linear, name="linear_e4m3_r262144_k1024_n4096", R=262144, K=1024, N=4096, dtype="e4m3",
             out="bf16", bias=True, act="silu"),
        # fp32 and odd sizes: logits over 509 tokens from rows of 1021
        dict(linear, name="linear_f32_r2000_k1021_n509", R=2000, K=1021, N=509, dtype="f32", out="f32",
             bias=True),
        # first position: one beam for each of 64 requests under the filter; latency
        dict(sample, name="sample_b64_m1_v512", B=64, M=1, V=512, dtype="bf16", top_p=0.9),
        # 64 x 4096 sampled continuations under the filter: the largest
        dict(sample, name="sample_b64_m4096_v512", B=64, M=4096, V=512, dtype="bf16", top_k=64,
             top_p=0.95, greedy=0.1),
        # fp32 logits, an odd vocabulary, no filter
        dict(sample, name="sample_f32_b16_m1000_v509", B=16, M=1000, V=509, dtype="f32", mask=False,
             top_k=50, min_p=0.05),
        # few rows over a large vocabulary
        dict(sample, name="sample_b32_m1_v128000", B=32, M=1, V=128000, dtype="bf16", mask=False,
             top_p=0.95, min_p=0.001),
    ]


def _log(rng, lo, hi):
    """A whole number of lo .. hi, its logarithm uniform."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _width(rng, lo, hi):
    """A row length: half of them multiples of 64 (of 16 below 64), the others any."""
    n = _log(rng, lo, hi)
    unit = 64 if n >= 64 else 16
    return max(unit, n // unit * unit) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["norm", "linear", "sample"])
    if op == "norm":
        D = _width(rng, 16, 8192)
        dtype = rng.choice(["f32", "bf16", "bf16"])
        return dict(op=op, R=_log(rng, 1, min(262144, (1 << 28) // D)), D=D, dtype=dtype,
                    out=rng.choice([dtype, "e4m3"]), residual=rng.random() < 0.7)
    if op == "linear":
        K, N = _width(rng, 16, 8192), _width(rng, 16, 8192)
        dtype = rng.choice(["f32", "bf16", "bf16", "e4m3", "e4m3"])
        R = _log(rng, 1, min(262144, (1 << 40) // (K * N), (1 << 30) // max(K, N)))
        return dict(op=op, R=R, K=K, N=N, dtype=dtype, out="f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]),
                    bias=rng.random() < 0.5, act=rng.choice(["none", "relu", "gelu", "silu"]),
                    residual=rng.random() < 0.5)
    V = _width(rng, 2, 131072)
    rows = _log(rng, 1, min(262144, (1 << 27) // V))
    B = rng.randint(1, min(64, rows))
    return dict(op=op, B=B, M=max(1, rows // B), V=V, dtype=rng.choice(["f32", "bf16", "bf16"]),
                mask=rng.random() < 0.5, top_k=rng.choice([0, 1, 20, 50, 100, 1000]),
                top_p=rng.choice([1.0, 0.5, 0.8, 0.9, 0.95, 0.99]), min_p=rng.choice([0.0, 0.0, 0.01, 0.1]),
                greedy=rng.choice([0.0, 0.1]))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _quantised(t):
    """Rows in e4m3 with their scales, as an 8-bit program holds its activations and weights."""
    scale = t.abs().amax(-1).clamp_min(TINY) / E4M3_MAX
    return (t / scale[:, None]).to(E4M3), scale


def prepare(case, seed):
    """Inputs, weights and the output buffers that a decode loop keeps."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, dev = case, "cuda"
    s = {"case": c}
    if c["op"] == "norm":
        dt, shape = DTYPES[c["dtype"]], (c["R"], c["D"])
        # a residual stream: rows of different sizes, a few dimensions far larger than the rest
        size = torch.exp(0.5 * _normal(g, c["R"], 1))
        s["x"] = (_normal(g, *shape) * size).to(dt)
        s["residual"] = None
        if c["residual"]:
            wide = torch.where(torch.rand(c["D"], generator=g, device=dev) < 0.01, 20.0, 1.0)
            s["residual"] = (_normal(g, *shape) * size * wide).to(dt)
        s["weight"] = (1 + 0.1 * _normal(g, c["D"])).to(dt)
        s["sum"] = torch.empty(shape, dtype=dt, device=dev) if c["residual"] else None
        s["out"] = torch.empty(shape, dtype=DTYPES[c["out"]], device=dev)
        s["scale"] = torch.empty(c["R"], device=dev) if c["out"] == "e4m3" else None
    elif c["op"] == "linear":
        dt, to = DTYPES[c["dtype"]], DTYPES[c["out"]]
        x, w = _normal(g, c["R"], c["K"]), _normal(g, c["N"], c["K"]) / math.sqrt(c["K"])
        s["x_scale"] = s["w_scale"] = None
        if c["dtype"] == "e4m3":
            (s["x"], s["x_scale"]), (s["w"], s["w_scale"]) = _quantised(x), _quantised(w)
        else:
            s["x"], s["w"] = x.to(dt), w.to(dt)
        s["bias"] = (0.1 * _normal(g, c["N"])).to(to) if c["bias"] else None
        s["residual"] = _normal(g, c["R"], c["N"]).to(to) if c["residual"] else None
        s["out"] = torch.empty((c["R"], c["N"]), dtype=to, device=dev)
    else:
        B, R, V = c["B"], c["B"] * c["M"], c["V"]
        s["logits"] = (3 * _normal(g, R, V)).to(DTYPES[c["dtype"]])
        s["uniform"] = torch.rand(R, generator=g, device=dev)
        s["prev"] = -3 * torch.rand(R, generator=g, device=dev)
        s["mask"] = None
        if c["mask"]:       # the filter lets six tokens of ten through, as packed words
            words = torch.zeros((R, (V + 31) // 32), dtype=torch.int32, device=dev)
            at = torch.arange(words.shape[1], device=dev) * 32
            for bit in range(32):
                on = (torch.rand(words.shape, generator=g, device=dev) < 0.6) & (at + bit < V)
                words |= on.to(torch.int32) << bit
            s["mask"] = words
        T = 0.5 + torch.rand(B, generator=g, device=dev)
        # some requests of a batch ask for the best token
        s["temperature"] = torch.where(torch.rand(B, generator=g, device=dev) < c["greedy"], torch.zeros_like(T), T)
        s["top_k"] = torch.full((B,), c["top_k"], dtype=torch.int32, device=dev) if c["top_k"] else None
        s["top_p"] = torch.full((B,), c["top_p"], device=dev) if c["top_p"] < 1 else None
        s["min_p"] = torch.full((B,), c["min_p"], device=dev) if c["min_p"] else None
        s["tokens"] = torch.empty(R, dtype=torch.int32, device=dev)
        s["scores"] = torch.empty(R, device=dev)
    return s


def _norm(s):
    h = s["x"].float()
    outs = []
    if s["residual"] is not None:
        h = h + s["residual"].float()
        outs.append(h.to(s["x"].dtype))
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    if s["scale"] is None:
        return outs + [y.to(s["x"].dtype)]
    scale = y.abs().amax(-1).clamp_min(TINY) / E4M3_MAX
    return outs + [(y / scale[:, None]).to(E4M3), scale]


def _act(y, act):
    if act == "relu":
        return y.clamp_min(0)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y / (1 + torch.exp(-y)) if act == "silu" else y


def _linear(s):
    y = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["x_scale"] is not None:
        y = y * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(s["out"].dtype)]


def _allowed(mask, V):
    v = torch.arange(V, device=mask.device)
    return (mask[:, v // 32] >> (v % 32)) & 1 != 0


def _sample(s):
    """In 64 bits: a token next to a border is decided by the last digits of long sums."""
    z, V, M = s["logits"].double(), s["case"]["V"], s["case"]["M"]
    each = lambda t: t.double().repeat_interleave(M)[:, None]  # noqa: E731
    top = z.amax(-1, keepdim=True)
    log_sum = top + torch.log(torch.exp(z - top).sum(-1, keepdim=True))
    cand = z if s["mask"] is None else torch.where(_allowed(s["mask"], V), z, -math.inf)
    ranked, order = torch.sort(cand, dim=-1, descending=True, stable=True)
    best = ranked[:, :1]
    T = each(s["temperature"])
    w = torch.exp((ranked - torch.where(best > -math.inf, best, torch.zeros_like(best))) / torch.where(T > 0, T, 1.0))
    rank = torch.arange(V, device=z.device)
    keep = (w > 0) & ((T > 0) | (rank == 0))
    if s["top_k"] is not None:
        keep = keep & (rank < each(s["top_k"]))
    w = torch.where(keep, w, 0.0)
    if s["top_p"] is not None:
        upto = torch.cumsum(w, -1)
        keep = keep & ((upto - w < each(s["top_p"]) * upto[:, -1:]) | (rank == 0))
    if s["min_p"] is not None:
        keep = keep & (w >= each(s["min_p"]))
    w = torch.zeros_like(z).scatter_(1, order, torch.where(keep, w, 0.0))
    upto = torch.cumsum(w, -1)
    hit = (upto > s["uniform"].double()[:, None] * upto[:, -1:]) & (w > 0)
    token = torch.argmax(hit.to(torch.int8), -1, keepdim=True)
    alive = best > -math.inf
    score = s["prev"].double()[:, None] + torch.gather(z, 1, token) - log_sum
    token = torch.where(alive, token, -1)
    return [token[:, 0].to(torch.int32), torch.where(alive, score, -math.inf)[:, 0].float()]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"norm": _norm, "linear": _linear, "sample": _sample}[c["op"]](s)
    from paper_2608_00938_amd import grace as G
    if c["op"] == "norm":
        G.grace_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], sum_out=s["sum"], out=s["out"],
                         out_scale=s["scale"])
        return [t for t in (s["sum"], s["out"], s["scale"]) if t is not None]
    if c["op"] == "linear":
        return [G.grace_linear(s["x"], s["w"], bias=s["bias"], act=c["act"], residual=s["residual"],
                               x_scale=s["x_scale"], w_scale=s["w_scale"], out=s["out"])]
    return list(G.grace_sample(s["logits"], s["uniform"], c["B"], c["M"], temperature=s["temperature"],
                               top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], mask=s["mask"],
                               prev_scores=s["prev"], tokens=s["tokens"], scores=s["scores"]))


def work(case):
    c = case
    if c["op"] == "norm":
        n = c["R"] * c["D"]
        size = BYTES[c["dtype"]]
        moved = n * (size * (3 if c["residual"] else 1) + BYTES[c["out"]]) + c["D"] * size
        return {"bytes": moved + (4 * c["R"] if c["out"] == "e4m3" else 0), "flops": 5 * n}
    if c["op"] == "linear":
        R, K, N, to = c["R"], c["K"], c["N"], BYTES[c["out"]]
        moved = (R + N) * K * BYTES[c["dtype"]] + R * N * to * (2 if c["residual"] else 1)
        moved += (N * to if c["bias"] else 0) + (4 * (R + N) if c["dtype"] == "e4m3" else 0)
        return {"bytes": moved, "flops": 2 * R * N * K}
    R, V = c["B"] * c["M"], c["V"]
    moved = R * V * BYTES[c["dtype"]] + (R * ((V + 31) // 32) * 4 if c["mask"] else 0) + 16 * R
    return {"bytes": moved, "flops": 12 * R * V}


def _exact_rows(s, lo, hi):
    """Tokens and scores of the rows lo .. hi by counting instead of ranking's sums: a token's
    place and the mass before it come from the sorted row, its own membership from these."""
    c = s["case"]
    V = c["V"]
    z = s["logits"][lo:hi].double()
    req = torch.arange(lo, hi, device=z.device) // c["M"]
    logp = z - torch.logsumexp(z, 1, keepdim=True)
    ok = torch.isfinite(z)
    if s["mask"] is not None:
        word = s["mask"][lo:hi].to(torch.int64) & 0xFFFFFFFF
        ok &= ((word[:, :, None] >> torch.arange(32, device=z.device)) & 1).flatten(1)[:, :V].bool()
    neg = torch.where(ok, -z, torch.full_like(z, math.inf))
    order = torch.argsort(neg, dim=1, stable=True)
    place = torch.empty_like(order).scatter_(1, order, torch.arange(V, device=z.device).expand_as(order))
    T = s["temperature"].double()[req][:, None]
    lowest = neg.amin(1, keepdim=True)
    e = torch.exp(-(neg - lowest) / T.clamp_min(1e-300))
    e = torch.where(ok & (T > 0), e, (place == 0).double() * ok)
    n = torch.full_like(T, V) if s["top_k"] is None else s["top_k"].double()[req][:, None]
    e = torch.where(place < n, e, torch.zeros_like(e))
    if s["top_p"] is not None:
        run_mass = torch.cumsum(torch.gather(e, 1, order), 1)
        left = s["top_p"].double()[req][:, None] * run_mass[:, -1:]
        count = (run_mass < left).sum(1, keepdim=True) + 1     # the shortest prefix that reaches it
        least = torch.where(place < count, e, torch.zeros_like(e))
    else:
        least = e
    if s["min_p"] is not None:
        least = torch.where(e >= s["min_p"].double()[req][:, None], least, torch.zeros_like(e))
    mass = torch.cumsum(least, 1)
    token = (mass <= s["uniform"][lo:hi].double()[:, None] * mass[:, -1:]).sum(1).clamp_max(V - 1)
    dead = ~ok.any(1)
    score = s["prev"][lo:hi].double() + torch.gather(logp, 1, token[:, None])[:, 0]
    return torch.where(dead, -1, token).to(torch.int32), torch.where(dead, -math.inf, score)


def exact(case, seed):
    """The definitions in 64 bits, on the inputs of ``prepare``."""
    s, c = prepare(case, seed), case
    if c["op"] == "norm":
        x, weight = s["x"].double(), s["weight"].double()
        outs = []
        if s["residual"] is not None:
            x = x + s["residual"].double()
            outs.append(x)
        y = weight * (x / torch.sqrt(x.square().sum(1, keepdim=True) / c["D"] + EPS))
        if c["out"] != "e4m3":
            return outs + [y]
        largest = torch.maximum(y.amax(1), -y.amin(1)).clamp_min(TINY)
        return outs + [y * (E4M3_MAX / largest[:, None]), largest / E4M3_MAX]
    if c["op"] == "linear":
        x, w = s["x"].double(), s["w"].double()
        if s["x_scale"] is not None:
            x, w = x * s["x_scale"].double()[:, None], w * s["w_scale"].double()[:, None]
        y = x @ w.t().contiguous()
        if s["bias"] is not None:
            y += s["bias"].double()
        if c["act"] == "relu":
            y = torch.where(y > 0, y, torch.zeros_like(y))
        elif c["act"] == "gelu":
            y = y * 0.5 * torch.special.erfc(-y / math.sqrt(2.0))
        elif c["act"] == "silu":
            y = y * torch.special.expit(y)
        return [y if s["residual"] is None else y + s["residual"].double()]
    R, step = c["B"] * c["M"], max(1, (1 << 24) // c["V"])
    parts = [_exact_rows(s, lo, min(R, lo + step)) for lo in range(0, R, step)]
    return [torch.cat(p) for p in zip(*parts)]
