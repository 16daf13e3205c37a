"""Performance cases of the operators around an attention layer whose projections run in 8-bit
floating point:

  quantize   e4m3 codes with one binary32 step for each 1 x 128 block of the activations, or for
             each 128 x 128 block of a weight
  linear     the product of such codes: Y = sum over blocks of step * step * (sum of code * code)
  rotate     the norm of every query and key head and the rotation by position, in one pass over
             the rows of a fused query/key/value projection; one or several position axes
  attend     softmax attention with grouped heads over packed sequences of different lengths,
             causal or not, from single tokens over a long cache to whole prompts

`own` chooses between the library's entry points and the plain form of the same operators in
elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

G = 128                      # channels (and, of a weight, outputs) that share one step
E4M3_MAX = 448.0
FLOOR = 1e-8                 # smallest magnitude that a step is made for
EPS = 1e-6
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


# --------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------
def _quantize(name, tile, rows, K, dtype):
    c = {"kind": "quantize", "tile": tile, "rows": rows, "K": K, "dtype": dtype}
    return dict(c, name=name) if name else c


def _linear(name, M, K, N, out, bias=False):
    c = {"kind": "linear", "M": M, "K": K, "N": N, "out": out, "bias": bias}
    return dict(c, name=name) if name else c


def _rotate(name, T, Hq, Hk, D, R, axes, interleaved, dtype, far=0):
    c = {"kind": "rotate", "T": T, "Hq": Hq, "Hk": Hk, "D": D, "R": R, "axes": axes,
         "interleaved": interleaved, "dtype": dtype, "far": far}
    return dict(c, name=name) if name else c


def _attend(name, S, q_lo, q_hi, ctx_lo, ctx_hi, causal, Hq, Hk, D, dtype):
    """S sequences; sequence i has between q_lo and q_hi queries and that many keys plus
    between ctx_lo and ctx_hi earlier ones."""
    c = {"kind": "attend", "S": S, "q_lo": q_lo, "q_hi": q_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
         "causal": causal, "Hq": Hq, "Hk": Hk, "D": D, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # The input of a last-stage projection, batch 8 of 11 x 11 tokens: nothing but latency.
        _quantize("quantize_stage4", "row", 968, 512, "f16"),
        # The widest activation of a transformer layer at batch 32 of 64 x 64 tokens.
        _quantize("quantize_wide", "row", 131072, 4096, "bf16"),
        # A weight, once when a model is loaded.
        _quantize("quantize_weight", "square", 4096, 1024, "f32"),
        # One token through one square layer: the weight is read and hardly anything computed.
        _linear("linear_one_token", 1, 4096, 4096, "bf16"),
        # The query projection of a last stage, batch 8 of 11 x 11 tokens.
        _linear("linear_stage4", 968, 512, 512, "f16", True),
        # Nothing a multiple of anything: odd rows, channels and outputs, a binary32 result.
        _linear("linear_ragged", 6845, 333, 777, "f32", True),
        # The expansion of an MLP at batch 32 of 64 x 64 tokens: the largest product.
        _linear("linear_fc1", 131072, 1024, 4096, "bf16"),
        # One step of 16 sequences that answer: grouped heads, positions far into the text.
        _rotate("rotate_step", 16, 32, 8, 128, 128, 1, False, "bf16", 30000),
        # 8 images of 64 x 64 tokens, positions in height and width, neighbouring pairs.
        _rotate("rotate_images", 32768, 16, 16, 64, 64, 2, True, "f16"),
        # A batch of small images or windows of 7 x 7 to 14 x 14 tokens, every token sees all.
        _attend("attend_windows", 64, 49, 196, 0, 0, False, 16, 16, 64, "f16"),
        # Prompts of different lengths packed into one call, causal, grouped heads.
        _attend("attend_prompts", 8, 311, 4096, 0, 0, True, 32, 8, 128, "bf16"),
        # One token each of 16 sequences over caches of different lengths.
        _attend("attend_step", 16, 1, 1, 4000, 32000, True, 32, 8, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    """Mostly multiples of 64 as layers have them, some of 8, some odd."""
    c, how = _log_int(rng, lo, hi), rng.random()
    return max(64, (c + 32) // 64 * 64) if how < 0.6 else max(8, c // 8 * 8) if how < 0.8 else c


def _heads(rng):
    Hk = rng.choice((1, 2, 4, 8, 16))
    return Hk * rng.choice((1, 2, 3, 4, 8) if Hk <= 4 else (1, 2, 4) if Hk == 8 else (1, 2)), Hk


def draw(rng):
    kind = rng.choice(("quantize", "linear", "linear", "rotate", "attend", "attend"))
    while True:
        if kind == "quantize":
            if rng.random() < 0.3:
                c = _quantize(None, "square", _channels(rng, 64, 8192), _channels(rng, 64, 8192),
                              rng.choice(("f32", "bf16", "f16")))
            else:
                c = _quantize(None, "row", _log_int(rng, 1, 131072), _channels(rng, 32, 8192),
                              rng.choice(("f16", "bf16", "f32")))
            fits = c["rows"] * c["K"] * SIZE[c["dtype"]] <= 1 << 30
        elif kind == "linear":
            M = _log_int(rng, 1, 64) if rng.random() < 0.35 else _log_int(rng, 64, 131072)
            c = _linear(None, M, _channels(rng, 32, 8192), _channels(rng, 32, 8192),
                        rng.choice(("f16", "bf16", "f32")), rng.random() < 0.5)
            fits = c["M"] * c["K"] * c["N"] <= 1 << 39 and c["M"] * c["N"] <= 1 << 28
        elif kind == "rotate":
            Hq, Hk = _heads(rng)
            D = rng.choice((32, 64, 64, 96, 128, 128, 256))
            R = D if rng.random() < 0.7 else max(16, D // 2 // 16 * 16)
            c = _rotate(None, _log_int(rng, 1, 65536), Hq, Hk, D, R, rng.choice((1, 1, 2, 3)),
                        rng.random() < 0.4, rng.choice(("f16", "bf16", "bf16", "f32")),
                        rng.choice((0, 0, 1000, 100000)))
            fits = c["T"] * (Hq + Hk) * D * SIZE[c["dtype"]] <= 1 << 27
        else:
            Hq, Hk = _heads(rng)
            D = rng.choice((32, 64, 64, 80, 96, 128, 128))
            dtype = rng.choice(("f16", "bf16"))
            form = rng.choice(("images", "prompts", "steps"))
            if form == "images":
                lo = _log_int(rng, 9, 700)
                c = _attend(None, _log_int(rng, 1, 128), lo, lo + rng.randint(0, 2 * lo), 0,
                            rng.choice((0, 0, 77)), False, Hq, Hk, D, dtype)
            elif form == "prompts":
                hi = _log_int(rng, 30, 4096)
                c = _attend(None, _log_int(rng, 1, 16), hi // rng.choice((1, 2, 10, 1000)), hi, 0,
                            rng.choice((0, 0, 500, 5000)), True, Hq, Hk, D, dtype)
            else:
                hi = _log_int(rng, 60, 32000)
                c = _attend(None, _log_int(rng, 1, 64), 1, rng.choice((1, 1, 1, 4)),
                            hi // rng.choice((1, 2, 20)), hi, True, Hq, Hk, D, dtype)
            w, most = work(c), work(listed()[10])
            ql, kl = _lengths(c)
            fits = (w["flops"] <= most["flops"] and w["bytes"] <= 1 << 30
                    and c["S"] * Hq * max(ql) * max(kl) <= 1 << 32)
        if fits:
            return c


def _spread(i, lo, hi):
    """The i-th of a fixed sequence of lengths from lo to hi, hi first."""
    return hi - (i * 7919) % (hi - lo + 1)


def _lengths(c):
    q = [_spread(i, c["q_lo"], c["q_hi"]) for i in range(c["S"])]
    return q, [n + _spread(i, c["ctx_lo"], c["ctx_hi"]) for i, n in enumerate(q)]


def _pairs_seen(ql, kl, causal):
    """(query, key) pairs: a causal query sees the keys up to its own place at the end."""
    return sum(q * k - (q * (q - 1) // 2 if causal else 0) for q, k in zip(ql, kl))


def work(case):
    c = case
    if c["kind"] == "quantize":
        n = c["rows"] * c["K"]
        steps = -(-c["K"] // G) * (c["rows"] if c["tile"] == "row" else -(-c["rows"] // G))
        return {"bytes": n * SIZE[c["dtype"]] + n + 4 * steps, "flops": 3 * n}
    if c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        KB, NB = -(-K // G), -(-N // G)
        return {"bytes": M * K + N * K + 4 * KB * (M + NB) + M * N * SIZE[c["out"]] + (4 * N if c["bias"] else 0),
                "flops": 2 * M * K * N}
    if c["kind"] == "rotate":
        n = c["T"] * (c["Hq"] + c["Hk"]) * c["D"]
        return {"bytes": 2 * n * SIZE[c["dtype"]] + 4 * c["T"] * c["axes"], "flops": 8 * n}
    ql, kl = _lengths(c)
    Tq, Tk, D, z = sum(ql), sum(kl), c["D"], SIZE[c["dtype"]]
    return {"bytes": z * D * (2 * Tq * c["Hq"] + 2 * Tk * c["Hk"]) + 4 * Tq * c["Hq"],
            "flops": 4 * D * c["Hq"] * _pairs_seen(ql, kl, c["causal"])}


# --------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------
def _activations(rows, K, g):
    """[rows, K] float32: a Laplace bulk, one row in twelve 20 times as wide."""
    u = torch.rand((rows, K), generator=g, device="cuda") - 0.5
    x = -torch.sign(u) * torch.log1p(-2.0 * u.abs().clamp_(max=0.4999999))
    wide = torch.rand((rows, 1), generator=g, device="cuda") < 1.0 / 12
    return x.mul_(torch.where(wide, 20.0, 1.0))


def _padded(codes):
    """e4m3 values as a program holds them: bytes, rows a multiple of 16 apart."""
    rows, K = codes.shape
    q = torch.zeros((rows, (K + 15) // 16 * 16), dtype=torch.uint8, device="cuda")
    q[:, :K] = codes.view(torch.uint8)
    return q


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(c)
    if c["kind"] == "quantize":
        x = _activations(c["rows"], c["K"], g)
        s["X"] = (x if c["tile"] == "row" else 0.02 * x).to(DT[c["dtype"]])
        rows, K = c["rows"], c["K"]
        s["Q"] = torch.empty((rows, (K + 15) // 16 * 16), dtype=torch.uint8, device="cuda")
        s["step"] = torch.empty((rows if c["tile"] == "row" else -(-rows // G), -(-K // G)), device="cuda")
    elif c["kind"] == "linear":
        s["Qx"], s["xs"] = _codes(_activations(c["M"], c["K"], g), 1)
        s["Qw"], s["ws"] = _codes(0.02 * randn(c["N"], c["K"]), G)
        s["Qx"], s["Qw"] = _padded(s["Qx"]), _padded(s["Qw"])
        s["b"] = 0.02 * randn(c["N"]) if c["bias"] else None
        s["Y"] = torch.empty((c["M"], c["N"]), dtype=DT[c["out"]], device="cuda")
    elif c["kind"] == "rotate":
        T, Hq, Hk, D, R, A = (c[k] for k in ("T", "Hq", "Hk", "D", "R", "axes"))
        qkv = (randn(T, Hq + 2 * Hk, D) * (0.5 + randn(T, 1, 1).abs())).to(DT[c["dtype"]])
        s["Qi"], s["Ki"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        s["wq"], s["wk"] = 1.0 + 0.1 * randn(D), 1.0 + 0.1 * randn(D)
        # pairs dealt to the axes in equal runs, frequencies falling within each run
        P, run = R // 2, -(-(R // 2) // A)
        at = torch.arange(P, device="cuda")
        s["axis"] = (at // run).to(torch.int32) if A > 1 else None
        s["freq"] = (10000.0 ** (-(at % run).double() / run)).float()
        t = torch.arange(T, device="cuda")
        side = max(1, math.isqrt(max(T // 8, 1)))
        place = [t % 4096 + c["far"]] if A == 1 else [t // side % side, t % side, t // (side * side)][:A]
        s["pos"] = (torch.stack(place) + torch.randint(0, 50, (A, 1), generator=g, device="cuda")).to(torch.int32)
        s["out"] = (torch.empty((T, Hq, D), dtype=qkv.dtype, device="cuda"),
                    torch.empty((T, Hk, D), dtype=qkv.dtype, device="cuda"))
    else:
        ql, kl = _lengths(c)
        Tq, Tk, Hq, Hk, D, dt = sum(ql), sum(kl), c["Hq"], c["Hk"], c["D"], DT[c["dtype"]]
        common = randn(1, 1, D)          # a direction that queries and keys share: uneven scores
        s["Qh"] = (randn(Tq, Hq, D) + 0.5 * common).to(dt)
        s["Kh"] = (randn(Tk, Hk, D) + randn(Tk, Hk, 1) * 0.5 * common).to(dt)
        s["Vh"] = (randn(Tk, Hk, D) + 0.2).to(dt)
        s["cu_q"], s["cu_k"] = _starts(ql), _starts(kl)
        s["most_q"], s["most_k"] = max(ql), max(kl)
        s["scale"] = 1.0 / math.sqrt(D)
        s["O"] = torch.empty((Tq, Hq, D), dtype=dt, device="cuda")
        s["lse"] = torch.empty((Tq, Hq), device="cuda")
        if own:                          # scratch of the split over a long cache, kept by the program
            from paper_2604_16855_amd import tdq
            n = tdq.tdq_attention_workspace_bytes(Tq, Tk, c["S"], Hq, Hk, D)
            s["work"] = torch.empty((max(n, 1),), dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------
def _codes(x, rows):
    """(e4m3 values, steps) of x[R, K], a step for each `rows` x 128 block."""
    R, K = x.shape
    RB, KB = -(-R // rows), -(-K // G)
    xp = torch.zeros((RB * rows, KB * G), device=x.device)
    xp[:R, :K] = x
    xp = xp.view(RB, rows, KB, G)
    most = xp.abs().amax(dim=(1, 3)).clamp(min=FLOOR)
    step = most / torch.full_like(most, E4M3_MAX)
    q = (xp / step[:, None, :, None]).view(RB * rows, KB * G)[:R, :K]
    return q.contiguous().to(torch.float8_e4m3fn), step


def _values(q, step, rows, K):
    """What padded codes and their steps stand for, float32 [R, K]."""
    full = step.repeat_interleave(rows, dim=0).repeat_interleave(G, dim=1)
    return q.view(torch.float8_e4m3fn)[:, :K].to(torch.float32) * full[:q.shape[0], :K]


def _linear_plain(s):
    y = _values(s["Qx"], s["xs"], 1, s["K"]) @ _values(s["Qw"], s["ws"], G, s["K"]).t().contiguous()
    return (y if s["b"] is None else y + s["b"]).to(DT[s["out"]])


def _rotate_heads(x, w, cos, sin, R, interleaved):
    x = x.float()
    y = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if interleaved else (y[..., :R // 2], y[..., R // 2:R])
    p, q = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((p, q), dim=-1).flatten(-2) if interleaved else torch.cat((p, q), dim=-1)
    return torch.cat((turned, y[..., R:]), dim=-1)


def _rotate_plain(s):
    axis = s["axis"].long() if s["axis"] is not None else torch.zeros_like(s["freq"], dtype=torch.long)
    angle = s["pos"].float()[axis] * s["freq"][:, None]
    cos, sin = angle.cos().t()[:, None], angle.sin().t()[:, None]
    dt = s["Qi"].dtype
    return (_rotate_heads(s["Qi"], s["wq"], cos, sin, s["R"], s["interleaved"]).to(dt),
            _rotate_heads(s["Ki"], s["wk"], cos, sin, s["R"], s["interleaved"]).to(dt))


def _attend_plain(s):
    """Every sequence padded to the longest, all scores at once."""
    Hq, Hk, D, S, mq, mk = s["Hq"], s["Hk"], s["D"], s["S"], s["most_q"], s["most_k"]
    dev, gr = s["Qh"].device, s["Hq"] // s["Hk"]
    q0, k0 = s["cu_q"][:-1].long(), s["cu_k"][:-1].long()
    nq, nk = s["cu_q"][1:].long() - q0, s["cu_k"][1:].long() - k0
    iq, ik = torch.arange(mq, device=dev), torch.arange(mk, device=dev)
    at_q = (q0[:, None] + iq).clamp(max=s["Qh"].shape[0] - 1)
    at_k = (k0[:, None] + ik).clamp(max=s["Kh"].shape[0] - 1)
    q = s["Qh"][at_q].float().view(S, mq, Hk, gr, D).permute(0, 2, 3, 1, 4).reshape(S * Hk, gr * mq, D)
    k = s["Kh"][at_k].float().permute(0, 2, 3, 1).reshape(S * Hk, D, mk).contiguous()
    v = s["Vh"][at_k].float().permute(0, 2, 1, 3).reshape(S * Hk, mk, D).contiguous()
    seen = (iq[None, :, None] < nq[:, None, None]) & (ik[None, None, :] < nk[:, None, None])
    if s["causal"]:
        seen = seen & (ik[None, None, :] <= iq[None, :, None] + (nk - nq)[:, None, None])
    z = (torch.bmm(q, k) * s["scale"]).view(S, Hk, gr, mq, mk)
    z = z.masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(dim=-1, keepdim=True)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = z.sub_(base).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.bmm(p.view(S * Hk, gr * mq, mk), v).view(S, Hk, gr, mq, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (base + total.log()).squeeze(-1)
    real = iq[None, :] < nq[:, None]
    o = o.permute(0, 3, 1, 2, 4).reshape(S, mq, Hq, D)[real]
    return o.to(s["Qh"].dtype), lse.permute(0, 3, 1, 2).reshape(S, mq, Hq)[real]


# --------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if not own:
        if kind == "quantize":
            return _codes(s["X"].float(), 1 if s["tile"] == "row" else G)
        return {"linear": _linear_plain, "rotate": _rotate_plain, "attend": _attend_plain}[kind](s)
    from paper_2604_16855_amd import tdq
    if kind == "quantize":
        f = tdq.tdq_quantize_act_f8 if s["tile"] == "row" else tdq.tdq_quantize_weight_f8
        q, step = f(s["X"], out=(s["Q"], s["step"]))
        return q[:, :s["K"]].view(torch.float8_e4m3fn), step
    if kind == "linear":
        return tdq.tdq_linear_f8(s["Qx"], s["xs"], s["K"], s["Qw"], s["ws"], bias=s["b"], out=s["Y"])
    if kind == "rotate":
        return tdq.tdq_norm_rotate(s["Qi"], s["Ki"], s["pos"], s["freq"], q_weight=s["wq"], k_weight=s["wk"],
                                   eps=EPS, axis=s["axis"], interleaved=s["interleaved"], out=s["out"])
    return tdq.tdq_attention(s["Qh"], s["Kh"], s["Vh"], s["cu_q"], s["cu_k"], scale=s["scale"],
                             causal=s["causal"], out=s["O"], lse=s["lse"], workspace=s["work"])


# --------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# --------------------------------------------------------------------------------------
def _nearest_e4m3(v):
    """v in float64 to the nearest value of sign, four exponent and three fraction bits (ties to even)."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    e = e + (v.abs() >= torch.exp2(e + 1)).double() - (v.abs() < torch.exp2(e)).double() * (e > -6).double()
    unit = torch.exp2(e - 3)
    return (torch.round(v / unit) * unit).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantize(s):
    rows, K, high = s["rows"], s["K"], 1 if s["tile"] == "row" else G
    X = s["X"]
    codes = torch.empty((rows, K), dtype=torch.float64, device="cuda")
    steps = torch.empty((-(-rows // high), -(-K // G)), dtype=torch.float64, device="cuda")
    for b in range(steps.shape[1]):
        x = X[:, b * G:(b + 1) * G].double()
        m = x.abs().amax(dim=1)
        pad = torch.zeros(steps.shape[0] * high, dtype=torch.float64, device="cuda")
        pad[:rows] = m
        steps[:, b] = pad.view(-1, high).amax(dim=1).clamp(min=FLOOR) / E4M3_MAX
        codes[:, b * G:(b + 1) * G] = _nearest_e4m3(x / steps[:, b].repeat_interleave(high)[:rows, None])
    return codes, steps


def _exact_linear(s):
    M, K, N = s["M"], s["K"], s["N"]
    w = s["Qw"].view(torch.float8_e4m3fn).to(torch.float64)
    y = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    out = torch.arange(N, device="cuda") // G
    for b in range(-(-K // G)):
        at = slice(b * G, min(K, (b + 1) * G))
        wb = (w[:, at] * s["ws"].double()[out, b][:, None]).t().contiguous()
        x = s["Qx"][:, at].contiguous().view(torch.float8_e4m3fn).to(torch.float64)
        y.addmm_(x * s["xs"][:, b:b + 1].double(), wb)
    return y if s["b"] is None else y + s["b"].double()


def _exact_rotate(s):
    D, R, P = s["D"], s["R"], s["R"] // 2
    which = [0] * P if s["axis"] is None else s["axis"].tolist()
    angle = torch.stack([s["pos"][which[p]].double() * s["freq"][p].double() for p in range(P)], dim=1)
    first = [2 * p if s["interleaved"] else p for p in range(P)]
    second = [2 * p + 1 if s["interleaved"] else p + P for p in range(P)]
    got = []
    for x, w in ((s["Qi"], s["wq"]), (s["Ki"], s["wk"])):
        x = x.double()
        n = (x * x).sum(dim=-1, keepdim=True) / D + EPS
        y = x / n.sqrt() * w.double()
        r = y.clone()
        c, d = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
        r[..., first] = y[..., first] * c - y[..., second] * d
        r[..., second] = y[..., first] * d + y[..., second] * c
        got.append(r)
    return tuple(got)


def _exact_attend(s):
    Hq, Hk, D = s["Hq"], s["Hk"], s["D"]
    o = torch.zeros(s["Qh"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    for i in range(s["S"]):
        nq, nk = cq[i + 1] - cq[i], ck[i + 1] - ck[i]
        if not nq or not nk:
            continue
        hide = (torch.arange(nk, device="cuda")[None, :]
                > torch.arange(nq, device="cuda")[:, None] + (nk - nq)) if s["causal"] else None
        for h in range(Hk):
            heads = slice(h * Hq // Hk, (h + 1) * Hq // Hk)
            q = s["Qh"][cq[i]:cq[i + 1], heads].double().transpose(0, 1).reshape(-1, D)
            k, v = (s[n][ck[i]:ck[i + 1], h].double() for n in ("Kh", "Vh"))
            z = ((q @ k.t().contiguous()) * s["scale"]).view(-1, nq, nk)
            if hide is not None:
                z = z.masked_fill(hide, -math.inf)
            l = torch.logsumexp(z, dim=-1)
            p = torch.exp(z - l.masked_fill(l == -math.inf, 0.0)[..., None])
            o[cq[i]:cq[i + 1], heads] = (p.view(-1, nk) @ v).view(-1, nq, D).transpose(0, 1)
            lse[cq[i]:cq[i + 1], heads] = l.t()
    return o, lse


def exact(case, seed):
    s = prepare(case, seed)
    return {"quantize": _exact_quantize, "linear": _exact_linear, "rotate": _exact_rotate,
            "attend": _exact_attend}[case["kind"]](s)
