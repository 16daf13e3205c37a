"""Oracles in 64 bits of the 8-bit linear, the head norm with rotation and the attention, straight from their
definitions, and the tolerances that follow from the types."""
import math

import torch

G = 128
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -149}


def dev():
    return torch.device("cuda:0")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, seed=0, dtype=torch.float32):
    return torch.randn(shape, generator=gen(seed), device="cuda").to(dtype)


# ---- codes -------------------------------------------------------------------------
def e4m3_table():
    """Values of the 256 codes (OCP e4m3: bias 7, no infinities, 0x7F and 0xFF NaN)."""
    t = []
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = math.nan if (c & 127) == 127 else (1 + f / 8) * 2.0 ** (e - 7) if e else f / 8 * 2.0 ** -6
        t.append(-v if c & 128 else v)
    return torch.tensor(t, dtype=torch.float64, device="cuda")


def code_values(q, K):
    return e4m3_table()[q[:, :K].long()]


def nearest_codes(v):
    """Codes of float32 values within the type's range: to nearest, ties to the even code."""
    table = e4m3_table()[:127]                              # magnitudes, ascending
    a = v.abs().double().contiguous()
    hi = torch.searchsorted(table, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - table[lo], table[hi] - a
    take_hi = (dh < dl) | ((dh == dl) & (hi % 2 == 0)) | (a <= 0)
    code = torch.where(take_hi, hi, lo)
    code = torch.where(a == 0, torch.zeros_like(code), code)
    return (code + 128 * torch.signbit(v).long()).to(torch.uint8)


def block_codes(x, rows):
    """(codes, steps) of float32 x[R, K] with a step for each rows x 128 block."""
    R, K = x.shape
    RB, KB = -(-R // rows), -(-K // G)
    pad = torch.zeros((RB * rows, KB * G), dtype=torch.float32, device=x.device)
    pad[:R, :K] = x
    pad = pad.view(RB, rows, KB, G)
    most = pad.abs().amax(dim=(1, 3)).clamp(min=1e-8)
    step = (most.double() / 448.0).float()                  # (the 64-bit quotient rounds as the 32-bit one)
    quotient = (pad.double() / step.double()[:, None, :, None]).float()
    return nearest_codes(quotient.view(RB * rows, KB * G)[:R, :K]), step


def linear(qx, xs, K, qw, ws, bias=None):
    """(Y, sum of the magnitudes of its terms) in 64 bits."""
    x, w = code_values(qx, K), code_values(qw, K)
    sx = xs.double().repeat_interleave(G, dim=1)[:, :K]
    sw = ws.double().repeat_interleave(G, dim=0).repeat_interleave(G, dim=1)[:w.shape[0], :K]
    X, Wt = x * sx, (w * sw).t().contiguous()
    y, mag = X @ Wt, X.abs() @ Wt.abs()
    return (y, mag) if bias is None else (y + bias.double(), mag + bias.double().abs())


# ---- norm and rotation -------------------------------------------------------------
def norm_rotate(x, w, eps, pos, freq, axis, interleaved):
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(dim=-1, keepdim=True) + eps).sqrt() * w.double()
    y = x.clone()
    P = 0 if freq is None else freq.numel()
    for p in range(P):
        row = 0 if axis is None else int(axis[p])
        # (the angle is a binary32 product by definition)
        a = (pos.view(-1, x.shape[0])[row].float() * freq[p]).double()[:, None]
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + P)
        y[..., i] = x[..., i] * a.cos() - x[..., j] * a.sin()
        y[..., j] = x[..., j] * a.cos() + x[..., i] * a.sin()
    return y


# ---- attention ---------------------------------------------------------------------
def starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def attention(Q, K, V, ql, kl, scale, causal):
    """(O, lse, tolerance of O, tolerance of lse) in 64 bits.

    Scores are binary32 sums of D exact products and one scaling: off by at most
    e = (D + 2) 2^-24 scale sum |q k|, which changes a weight by a factor exp(e).  A probability is rounded to the
    type of V (u relative, or half of its smallest number absolute, against a sum of at least about 1), the result once
    more; exponentials, sums and the rescaling of O are binary32 (a few units each and one for each of 64 keys)."""
    Tq, Hq, D = Q.shape
    Hk = K.shape[1]
    g = Hq // Hk
    O = torch.zeros((Tq, Hq, D), dtype=torch.float64, device=Q.device)
    L = torch.full((Tq, Hq), -math.inf, dtype=torch.float64, device=Q.device)
    tO, tL = torch.zeros_like(O), torch.zeros_like(L)
    u, tiny = UNIT[Q.dtype], TINY[Q.dtype]
    q0 = k0 = 0
    for nq, nk in zip(ql, kl):
        if nq and nk:
            for h in range(Hq):
                q, k, v = Q[q0:q0 + nq, h].double(), K[k0:k0 + nk, h // g].double(), V[k0:k0 + nk, h // g].double()
                kt = k.t().contiguous()
                s, off = (q @ kt) * scale, (q.abs() @ kt.abs()) * abs(scale) * (D + 2) * 2.0 ** -24
                if causal:
                    hide = (torch.arange(nk, device=s.device)[None, :]
                            > torch.arange(nq, device=s.device)[:, None] + (nk - nq))
                    s = s.masked_fill(hide, -math.inf)
                    off = off.masked_fill(hide, 0.0)
                lse = torch.logsumexp(s, dim=-1)
                w = torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
                e = off.amax(dim=-1, keepdim=True)
                more = u + 2 * e + (nk / 64 + 8) * 2.0 ** -23
                O[q0:q0 + nq, h] = w @ v
                tO[q0:q0 + nq, h] = (u * (w @ v).abs() + more * (w @ v.abs())
                                     + 2 * tiny * (1 + v.abs().sum(dim=0)))
                L[q0:q0 + nq, h] = lse
                tL[q0:q0 + nq, h] = e[:, 0] + (nk / 64 + 8) * 2.0 ** -23 + 4 * 2.0 ** -24 * lse.masked_fill(lse == -math.inf, 0.0).abs()
        q0 += nq
        k0 += nk
    return O, L, tO, tL


def check_attention(got, want):
    O, lse = got
    rO, rL, tO, tL = want
    assert torch.isfinite(O.double()).all()
    bad = (O.double() - rO).abs() / (tO + 1e-300)
    bad = bad.masked_fill((O.double() == rO), 0.0)
    assert float(bad.max()) <= 1.0, float(bad.max())
    empty = rL == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert bool((O[empty] == 0).all())
    if (~empty).any():
        d = ((lse.double() - rL).abs() / tL)[~empty]
        assert float(d.max()) <= 1.0, float(d.max())
