"""Caches in pages and oracles in 64 bits of the operators on them, straight from their definitions."""
import math

import torch

import layer_util as L


class Cache:
    """Keys and values of sequences of these lengths in pages that lie anywhere in a larger cache; `K` and `V` are the
    sequences' own, one after the other.  Rows of the cache that no sequence uses hold `rest`."""

    def __init__(self, lengths, P, Hk, D, dtype, seed=0, rest=0.0, columns=None, spare=3, values=None):
        need = [-(-n // P) for n in lengths]
        self.P, self.lengths, n = P, list(lengths), sum(need) + spare
        ids = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
        columns = max([1] + need) if columns is None else columns
        self.lines = [[ids.pop() for _ in range(m)] for m in need]
        self.table = torch.tensor([r + [-1] * (columns - len(r)) for r in self.lines], dtype=torch.int32, device="cuda")
        self.len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.k = torch.full((n, P, Hk, D), rest, dtype=dtype, device="cuda")
        self.v = torch.full((n, P, Hk, D), rest, dtype=dtype, device="cuda")
        self.K, self.V = values or ([L.randn(m, Hk, D, seed=seed + 7 * i + 1, dtype=dtype) for i, m in enumerate(lengths)],
                                    [(L.randn(m, Hk, D, seed=seed + 7 * i + 2) + 0.3).to(dtype)
                                     for i, m in enumerate(lengths)])
        for line, K, V in zip(self.lines, self.K, self.V):
            for b, page in enumerate(line):
                part = slice(b * P, min((b + 1) * P, K.shape[0]))
                m = part.stop - part.start
                self.k[page, :m], self.v[page, :m] = K[part], V[part]


def masked(Q, K, V, seen, scale):
    """(O, lse, tolerance of O, tolerance of lse) in 64 bits of queries Q[n, Hq, D] over K, V[m, Hk, D] where seen
    [n, Hk, m].

    Tolerances as in layer_util.attention: scores are binary32 sums of D exact products and one scaling, off by at most
    e = (D + 2) 2^-24 scale sum |q k|, which changes a weight by a factor exp(e); a probability is rounded to the type
    of V (u relative, or half of its smallest number absolute, against a sum of about 1 at least), the result once
    more; exponentials, sums, the rescaling of O and the joining of parts are binary32: a few units each and one for
    each of 64 keys."""
    n, Hq, D = Q.shape
    m, Hk = K.shape[0], K.shape[1]
    g, u, tiny = Hq // Hk, L.UNIT[Q.dtype], L.TINY[Q.dtype]
    O = torch.zeros((n, Hq, D), dtype=torch.float64, device=Q.device)
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64, device=Q.device)
    tO, tL = torch.zeros_like(O), torch.zeros_like(lse)
    if n == 0 or m == 0:
        return O, lse, tO, tL
    for h in range(Hq):
        see = seen[:, h // g]
        q, k, v = Q[:, h].double(), K[:, h // g].double(), V[:, h // g].double()
        kt = k.t().contiguous()
        s = ((q @ kt) * scale).masked_fill(~see, -math.inf)
        off = ((q.abs() @ kt.abs()) * abs(scale) * (D + 2) * 2.0 ** -24).masked_fill(~see, 0.0)
        l = torch.logsumexp(s, dim=-1)
        w = torch.exp(s - l.masked_fill(l == -math.inf, 0.0)[:, None])
        e = off.amax(dim=-1, keepdim=True)
        more = u + 2 * e + (m / 64 + 8) * 2.0 ** -23
        O[:, h] = w @ v
        # (a row that sees nothing is 0 exactly)
        tO[:, h] = (u * (w @ v).abs() + more * (w @ v.abs()) + 2 * tiny * (1 + v.abs().sum(dim=0))) * see.any(dim=1)[:, None]
        lse[:, h] = l
        tL[:, h] = e[:, 0] + (m / 64 + 8) * 2.0 ** -23 + 4 * 2.0 ** -24 * l.masked_fill(l == -math.inf, 0.0).abs()
    return O, lse, tO, tL


def sequences(Q, ql, cache, scale, causal=True, prefixes=None, of=None, hidden=None):
    """The attention of packed queries over the sequences of a cache, prefix of[s] (None: none) of another in front;
    hidden[s]: keys of the sequence that nobody sees."""
    out, t = [], 0
    for s, (n, m) in enumerate(zip(ql, cache.lengths)):
        K, V = cache.K[s], cache.V[s]
        j = torch.arange(m, device="cuda")
        last = torch.arange(n, device="cuda") + (m - n) if causal else torch.full((n,), m, device="cuda")
        see = j[None, :] <= last[:, None]
        if hidden is not None and hidden[s] is not None:
            see = see & ~hidden[s][None, :]
        if prefixes is not None and of[s] is not None:
            p = of[s]
            K, V = torch.cat((prefixes.K[p], K)), torch.cat((prefixes.V[p], V))
            see = torch.cat((torch.ones((n, prefixes.lengths[p]), dtype=torch.bool, device="cuda"), see), dim=1)
        out.append(masked(Q[t:t + n], K, V, see[:, None].expand(-1, K.shape[1], -1), scale))
        t += n
    return tuple(torch.cat(x) for x in zip(*out))


def merged(a, b):
    """Two caches in one: (keys, values, table of a, table of b)."""
    n = a.k.shape[0]
    return torch.cat((a.k, b.k)), torch.cat((a.v, b.v)), a.table, torch.where(b.table >= 0, b.table + n, -1)


def best(score, there, always, count):
    """The pages of one row by the definition: numbers in a list, lowest first, -1 behind them."""
    order = sorted((b for b in range(len(score)) if there[b]),
                   key=lambda b: (not always[b], not math.isnan(score[b]), 0.0 if math.isnan(score[b]) else -score[b], b))
    take = sorted(order[:count])
    return take + [-1] * (count - len(take))
