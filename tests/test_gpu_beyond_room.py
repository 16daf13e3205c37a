"""Sequences of more keys than their line of the table has room for: query i of n is key len - n + i for every operator,
whether that key has a place or not."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L
import pages_util as U
from test_gpu_pages import _choice

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]
BIG = (1 << 31) - 1
# new tokens and keys of each sequence, pages of a line, keys of a page
CASES = [([20], [40], 2, 16), ([20, 3, 1], [40, 33, 500], 2, 16), ([5], [BIG], 3, 16), ([40], [70], 2, 16),
         ([100, 30], [150, 20], 6, 16), ([200], [300], 4, 64), ([300, 1, 7], [1000, 900, 513], 8, 64), ([50], [60], 1, 16),
         ([9, 0, 4], [12, 99, -7], 2, 16), ([130, 2], [BIG, 1 << 30], 1, 1024), ([700], [600], 16, 32),
         ([3] * 300, [14 + i % 9 for i in range(300)], 1, 16)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cache(lens, P, columns, Hk, D, dtype, seed=0):
    return U.Cache([min(max(m, 0), P * columns) for m in lens], P, Hk, D, dtype, seed=seed, rest=math.nan, columns=columns)


def _sees(ql, lens, room, causal):
    """Keys that each token sees."""
    out = []
    for n, m in zip(ql, lens):
        m = max(m, 0)
        out += [max(0, min(m - n + i + 1 if causal else m, room)) for i in range(n)]
    return out


def _attention(Q, ql, lens, c, room, causal, Hk, prefix=None, pages=None):
    """From the definition; a prefix's keys and values in front of all sequences; of each line's pages only the first."""
    sees, out, t = torch.tensor(_sees(ql, lens, room, causal), device="cuda"), [], 0
    for n, K, V in zip(ql, c.K, c.V):
        see = torch.arange(K.shape[0], device="cuda") < sees[t:t + n, None]
        if pages is not None:
            see = see & (torch.arange(K.shape[0], device="cuda") < pages * c.P)
        if prefix is not None:
            K, V = torch.cat((prefix[0], K)), torch.cat((prefix[1], V))
            see = torch.cat((torch.ones((n, prefix[0].shape[0]), dtype=torch.bool, device="cuda"), see), dim=1)
        out.append(U.masked(Q[t:t + n], K, V, see[:, None].expand(-1, Hk, -1), 1 / math.sqrt(Q.shape[2])))
        t += n
    return tuple(torch.cat(x) for x in zip(*out))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (8, 1, 128), (2, 2, 200)])
def test_attention(Hq, Hk, D, dtype, causal):
    for ql, lens, columns, P in CASES:
        print(f"[room] {ql[:4]} {lens[:4]} {columns} pages of {P} {Hq}/{Hk} D={D} {dtype} causal={causal}", flush=True)
        c, room = _cache(lens, P, columns, Hk, D, dtype), columns * P
        Q, cu = L.randn(sum(ql), Hq, D, seed=3, dtype=dtype), L.starts(ql)
        want = _attention(Q, ql, lens, c, room, causal, Hk)
        L.check_attention(tdq.tdq_attention_paged(Q, c.k, c.v, cu, c.table, _i32(lens), causal=causal, want_lse=True), want)
        for named in (columns, 1):
            chosen = torch.arange(named, dtype=torch.int32, device="cuda").expand(sum(ql), Hk, named).contiguous()
            L.check_attention(tdq.tdq_attention_selected(Q, c.k, c.v, chosen, cu, c.table, _i32(lens), causal=causal,
                                                         want_lse=True),
                              _attention(Q, ql, lens, c, room, causal, Hk, pages=named))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_behind_a_prefix(dtype):
    Hq, Hk, D = 4, 2, 64
    for ql, lens, columns, P in CASES:
        c, p = _cache(lens, P, columns, Hk, D, dtype), _cache([5 * P], P, 3, Hk, D, dtype, seed=50)
        k, v, table, pre_table = U.merged(c, p)
        Q = L.randn(sum(ql), Hq, D, seed=3, dtype=dtype)
        got = tdq.tdq_attention_paged(Q, k, v, L.starts(ql), table, _i32(lens), want_lse=True,
                                      prefix=(_i32([0, len(ql)]), pre_table, _i32([5 * P])))
        L.check_attention(got, _attention(Q, ql, lens, c, columns * P, True, Hk, prefix=(p.K[0], p.V[0])))


def _bounds_of(n, Hk, D, dtype):
    mid, wide = L.randn(n, Hk, D, seed=1), 1 + L.randn(n, Hk, D, seed=2).abs()
    return (mid - wide).to(dtype), (mid + wide).to(dtype)


def _check_choice(ql, lens, columns, P, Hq, Hk, D, dtype, count, causal):
    table = torch.randperm(len(ql) * columns, generator=torch.Generator().manual_seed(1)).view(len(ql), columns)
    table = table.to(torch.int32).cuda()
    lo, hi = _bounds_of(table.numel(), Hk, D, dtype)
    Q, sees = L.randn(sum(ql), Hq, D, seed=3, dtype=dtype), _sees(ql, lens, columns * P, causal)
    got = tdq.tdq_select_pages(Q, lo, hi, L.starts(ql), table, _i32(lens), P, count, causal=causal)
    # (each token by itself, as the last one of a sequence of what it sees)
    lines = table.repeat_interleave(torch.tensor(ql, device="cuda"), dim=0)
    want = _choice(Q, lo, hi, [1] * sum(ql), sees, lines, P, count, 1, 1, True)
    assert torch.equal(got, want), (got != want).nonzero()[:5].tolist()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
def test_choice(dtype, causal):
    for ql, lens, columns, P in CASES:
        print(f"[room] choice {ql[:4]} {lens[:4]} {columns} pages of {P} {dtype} causal={causal}", flush=True)
        _check_choice(ql, lens, columns, P, 4, 2, 64, dtype, 4, causal)
    _check_choice([3, 2], [16 * 700 + 1, BIG], 700, 16, 4, 2, 64, dtype, 90, causal)      # (more pages than a workgroup scores)
    _check_choice([260], [16 * 20 + 100], 20, 16, 32, 32, 16, dtype, 5, causal)           # (tokens of a sequence together)
    _check_choice([200, 100], [BIG, 16 * 9 + 70], 9, 16, 64, 32, 32, dtype, 4, causal)


def test_bounds_of_the_pages_of_new_tokens():
    """The pages that the queries' keys lie in, as far as they have a place, and no others."""
    P, Hk, D, dtype = 16, 2, 64, torch.bfloat16
    for n, m, columns, pages in ((20, 40, 2, [1]), (20, 33, 2, [0, 1]), (5, 100, 2, []), (40, BIG, 3, []), (3, 48, 3, [2]),
                                 (90, 100, 4, [0, 1, 2, 3]), (33, 80, 4, [2, 3])):
        c = _cache([m], P, columns, Hk, D, dtype)
        old = tuple(L.randn(c.k.shape[0], Hk, D, seed=s, dtype=dtype) for s in (8, 9))
        want, got = tuple(x.clone() for x in old), tuple(x.clone() for x in old)
        for b in pages:
            k = c.K[0][b * P:(b + 1) * P]
            want[0][c.lines[0][b]], want[1][c.lines[0][b]] = k.amin(dim=0), k.amax(dim=0)
        tdq.tdq_page_bounds(c.k, c.table, _i32([m]), cu_q=L.starts([n]), Tq=n, out=got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (n, m, columns)


@pytest.mark.parametrize("n", [6, 40, 300])
def test_a_token_sees_what_was_written_for_it(n):
    """Keys written by append, then attended to: the token's own key is the last one that it sees."""
    P, columns, Hk, D, have, dtype = 16, 3, 1, 64, 30, torch.float16
    room = P * columns
    K, V = L.randn(have + n, Hk, D, seed=1, dtype=dtype), L.randn(have + n, Hk, D, seed=2, dtype=dtype)
    Q, table = L.randn(n, 4, D, seed=3, dtype=dtype), _i32([[4, 0, 2]])
    k, v = (torch.full((5, P, Hk, D), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    tdq.tdq_cache_append(None, K[:have], V[:have], k, v, L.starts([have]), table, _i32([have]))
    tdq.tdq_cache_append(None, K[have:], V[have:], k, v, L.starts([n]), table, _i32([have + n]))
    c = U.Cache.__new__(U.Cache)
    c.P, c.K, c.V = P, [K[:room]], [V[:room]]
    want = _attention(Q, [n], [have + n], c, room, True, Hk)
    chosen = torch.arange(columns, dtype=torch.int32, device="cuda").expand(n, Hk, columns).contiguous()
    cu, m = L.starts([n]), _i32([have + n])
    L.check_attention(tdq.tdq_attention_paged(Q, k, v, cu, table, m, want_lse=True), want)
    L.check_attention(tdq.tdq_attention_selected(Q, k, v, chosen, cu, table, m, want_lse=True), want)
