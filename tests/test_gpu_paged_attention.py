"""Softmax attention over a cache in pages, against 64 bits: whole sequences, shared prefixes, chosen pages."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L
import pages_util as U

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]
HEADS = [(1, 1, 64), (4, 2, 128), (6, 2, 32), (3, 1, 80), (8, 1, 96), (2, 2, 256), (5, 5, 8), (7, 1, 40), (2, 1, 200), (4, 2, 184)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _paged(ql, lens, P, Hq, Hk, D, dtype, causal=True, scale=None, seed=0, rest=float("nan"), **kw):
    c = U.Cache(lens, P, Hk, D, dtype, seed=seed, rest=rest)
    Q = L.randn(sum(ql), Hq, D, seed=seed + 100, dtype=dtype)
    got = tdq.tdq_attention_paged(Q, c.k, c.v, L.starts(ql), c.table, c.len, scale=scale, causal=causal, want_lse=True)
    L.check_attention(got, U.sequences(Q, ql, c, 1 / math.sqrt(D) if scale is None else scale, causal))


LENGTHS = [([1], [1]), ([5], [5]), ([64], [64]), ([65], [65]), ([33, 1, 200], [33, 1, 200]),
           ([0, 7, 0, 130, 0], [0, 7, 0, 130, 0]), ([3, 40, 1], [100, 41, 700]), ([129, 300], [129, 555])]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D", HEADS)
def test_lengths(Hq, Hk, D, dtype, causal):
    for i, (ql, lens) in enumerate(LENGTHS):
        P = (16, 32, 64, 256)[i % 4]
        print(f"[paged] {ql} {lens} P={P} {Hq}/{Hk} D={D} {dtype} causal={causal}", flush=True)
        _paged(ql, lens, P, Hq, Hk, D, dtype, causal, seed=i)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ql,lens,Hq,Hk,D", [([1] * 5, [1, 63, 64, 65, 3001], 32, 8, 128), ([1], [9000], 8, 8, 64),
                                             ([1, 1, 0, 1], [0, 17, 5, 2000], 4, 1, 128),
                                             ([4, 2, 1], [4, 1000, 333], 16, 2, 64), ([1] * 130, list(range(130)), 2, 1, 32),
                                             ([1], [5000], 40, 1, 128), ([1, 1], [4097, 12], 6, 2, 256),
                                             ([1, 300, 1], [2500, 900, 3], 8, 2, 64), ([9], [6000], 32, 8, 128)])
def test_single_tokens(ql, lens, Hq, Hk, D, dtype):
    for P in (16, 64):
        print(f"[paged] step {ql[:9]} {lens[:9]} P={P} {Hq}/{Hk} D={D} {dtype}", flush=True)
        for causal in (True, False):
            _paged(ql, lens, P, Hq, Hk, D, dtype, causal, seed=3)


@pytest.mark.parametrize("dtype", TYPES)
def test_prompts(dtype):
    _paged([1000, 17, 2049], [1000, 17, 2049], 64, 8, 2, 128, dtype)
    _paged([700, 300], [1900, 301], 16, 4, 4, 64, dtype)
    _paged([512, 100], [77, 1500], 32, 4, 2, 64, dtype, causal=False)
    _paged([1500], [1500], 128, 12, 1, 64, dtype)


@pytest.mark.parametrize("causal", [False, True])
def test_queries_that_see_no_key(causal):
    _paged([10, 70, 5], [4, 3, 0], 16, 4, 2, 64, torch.float16, causal)
    _paged([200], [130], 32, 2, 1, 128, torch.bfloat16, causal)
    _paged([700], [130], 32, 4, 1, 128, torch.bfloat16, causal)
    _paged([1, 9], [0, 0], 16, 2, 2, 64, torch.float16, causal)


def test_many_sequences():
    n = 3000
    ql, lens = [(i * 7) % 4 for i in range(n)], [(i * 5) % 39 for i in range(n)]
    c = U.Cache(lens, 16, 1, 32, torch.float16)
    Q = L.randn(sum(ql), 2, 32, seed=5, dtype=torch.float16)
    cu = L.starts(ql)
    O, lse = tdq.tdq_attention_paged(Q, c.k, c.v, cu, c.table, c.len, causal=False, want_lse=True)
    at = cu.tolist()
    for i in [0, 1, 2, 63, 64, 255, 256, 257, 1023, 1024, 1025, 2047, 2999, 2998, 2997]:
        one = U.Cache([lens[i]], 16, 1, 32, torch.float16, values=([c.K[i]], [c.V[i]]))
        a = slice(at[i], at[i + 1])
        if ql[i]:
            L.check_attention((O[a], lse[a]), U.sequences(Q[a], [ql[i]], one, 1 / math.sqrt(32), False))


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    _paged([50, 1], [50, 400], 16, 4, 2, 64, torch.float16, True, scale=scale)


def test_large_and_growing_scores():
    """Scores of hundreds, the largest key last or first, so that the running maximum moves all the time or never."""
    n, D = 700, 64
    Q = L.randn(40, 2, D, seed=1, dtype=torch.bfloat16).abs()
    V = L.randn(n, 1, D, seed=2, dtype=torch.bfloat16)
    up = torch.linspace(-3, 3, n, device="cuda")
    for ramp in (up, -up, up * 0):
        K = (ramp[:, None, None] * torch.ones((n, 1, D), device="cuda")).bfloat16()
        c = U.Cache([n], 16, 1, D, torch.bfloat16, values=([K], [V]))
        for scale in (1.0, 0.05):
            for ql in ([40], [1]):
                q = Q[:ql[0]]
                got = tdq.tdq_attention_paged(q, c.k, c.v, L.starts(ql), c.table, c.len, scale=scale, want_lse=True)
                L.check_attention(got, U.sequences(q, ql, c, scale))


def test_pages_that_are_not_there():
    """Keys in pages that are not there are seen by nobody; a line of nothing else gives zeros."""
    for ql, lens, P in (([1, 3], [500, 90], 16), ([40, 200], [500, 330], 32), ([1], [3000], 64)):
        c = U.Cache(lens, P, 2, 64, torch.float16, rest=float("nan"))
        hidden = []
        for s, m in enumerate(lens):
            h = torch.zeros(m, dtype=torch.bool, device="cuda")
            for b, bad in ((1, -1), (2, c.k.shape[0]), (4, 1 << 30), (len(c.lines[s]) - 1, -(1 << 31))):
                if b < len(c.lines[s]):
                    c.table[s, b] = bad
                    h[b * P:(b + 1) * P] = True
            hidden.append(h)
        Q = L.randn(sum(ql), 4, 64, seed=4, dtype=torch.float16)
        got = tdq.tdq_attention_paged(Q, c.k, c.v, L.starts(ql), c.table, c.len, want_lse=True)
        L.check_attention(got, U.sequences(Q, ql, c, 0.125, hidden=hidden))
        got = tdq.tdq_attention_paged(Q, c.k, c.v, L.starts(ql), c.table * 0 - 1, c.len, want_lse=True)
        assert bool((got[0] == 0).all()) and bool((got[1] == -math.inf).all())


def test_lengths_beyond_the_room_of_a_line():
    c = U.Cache([64, 30], 16, 2, 64, torch.bfloat16)
    Q = L.randn(2, 4, 64, seed=4, dtype=torch.bfloat16)
    want = tdq.tdq_attention_paged(Q, c.k, c.v, L.starts([1, 1]), c.table, c.len, want_lse=True)
    for big in (65, 1 << 30, (1 << 31) - 1):
        got = tdq.tdq_attention_paged(Q, c.k, c.v, L.starts([1, 1]), c.table, _i32([big, 30]), want_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = tdq.tdq_attention_paged(Q, c.k, c.v, L.starts([1, 1]), c.table, _i32([-5, 30]), want_lse=True)
    assert bool((got[0][0] == 0).all()) and bool((got[1][0] == -math.inf).all()) and torch.equal(got[0][1], want[0][1])


def test_rows_of_no_sequence_are_left():
    c = U.Cache([300, 20], 16, 2, 64, torch.float16)
    for ql, first in (([1, 2], 3), ([100, 2], 5)):
        Q = L.randn(first + sum(ql) + 40, 4, 64, seed=4, dtype=torch.float16)
        out = torch.full_like(Q, 9.0)
        lse = torch.full((Q.shape[0], 4), 9.0, device="cuda")
        cu = first + L.starts(ql)
        pre = U.Cache([70], 16, 2, 64, torch.float16, seed=50)
        k, v, own, table = U.merged(c, pre)
        for prefix in (None, (_i32([0, 1]), table, pre.len)):
            tdq.tdq_attention_paged(Q, k, v, cu, own, c.len, prefix=prefix, out=out, lse=lse)
            for x in (out, lse):
                assert bool((x[:first] == 9).all()) and bool((x[first + sum(ql):] == 9).all())
            part = slice(first, first + sum(ql))
            want = U.sequences(Q[part], ql, c, 0.125, prefixes=pre, of=[0 if prefix else None, None])
            L.check_attention((out[part], lse[part]), want)


# ---- prefixes ----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 128), (3, 1, 80), (8, 1, 64), (2, 2, 256), (16, 2, 32)])
def test_prefixes(Hq, Hk, D, dtype):
    cases = [([1] * 6, [1, 5, 100, 17, 0, 64], [1000], [0, 6]),
             ([1, 3, 2, 0, 50], [1, 3, 90, 5, 50], [70, 333], [0, 3, 5]),
             ([40, 200, 1], [40, 500, 1], [0, 129, 17], [0, 1, 2, 3]),
             ([2, 1, 1, 4], [2, 400, 31, 4], [500], [1, 3]),              # the first and the last have none
             ([5, 3], [2, 0], [300], [0, 2]),                            # fewer own keys than queries
             ([1] * 40, [i % 7 for i in range(40)], [2000, 65], [0, 25, 40]),
             ([1, 1], [9, 9], [50, 60], [0, 0, 2])]                      # a prefix of no sequence
    for i, (ql, lens, pre, first) in enumerate(cases):
        P = (16, 64, 32)[i % 3]
        print(f"[paged] prefixes {ql[:8]} {lens[:8]} {pre} P={P} {Hq}/{Hk} D={D} {dtype}", flush=True)
        own = U.Cache(lens, P, Hk, D, dtype, seed=i, rest=float("nan"))
        p = U.Cache(pre, P, Hk, D, dtype, seed=i + 50, rest=float("nan"))
        k, v, table, pre_table = U.merged(own, p)
        of = [next((g for g in range(len(pre)) if first[g] <= s < first[g + 1]), None) for s in range(len(ql))]
        Q = L.randn(sum(ql), Hq, D, seed=9, dtype=dtype)
        for causal in (True, False):
            got = tdq.tdq_attention_paged(Q, k, v, L.starts(ql), table, own.len, prefix=(_i32(first), pre_table, p.len),
                                          causal=causal, want_lse=True)
            L.check_attention(got, U.sequences(Q, ql, own, 1 / math.sqrt(D), causal, p, of))


def test_a_prefix_is_the_same_as_its_pages_in_every_line():
    """Sequences behind a prefix of whole pages, and the same keys through their own lines."""
    P, Hk, D, dtype = 16, 2, 64, torch.bfloat16
    ql, lens = [1, 4, 30, 1], [1, 70, 30, 200]
    own, pre = U.Cache(lens, P, Hk, D, dtype), U.Cache([64], P, Hk, D, dtype, seed=50)
    k, v, table, pre_table = U.merged(own, pre)
    Q = L.randn(sum(ql), 4, D, seed=1, dtype=dtype)
    want = U.sequences(Q, ql, own, 0.125, True, pre, [0] * 4)
    whole = torch.cat((pre_table.expand(4, -1), table), dim=1).contiguous()
    for got in (tdq.tdq_attention_paged(Q, k, v, L.starts(ql), table, own.len, prefix=(_i32([0, 4]), pre_table, pre.len), want_lse=True),
                tdq.tdq_attention_paged(Q, k, v, L.starts(ql), whole, own.len + 64, want_lse=True)):
        L.check_attention(got, want)


# ---- chosen pages ------------------------------------------------------------------
def _chosen(ql, lens, P, Hq, Hk, D, dtype, count, causal=True, seed=0, pick=None, scale=None):
    c = U.Cache(lens, P, Hk, D, dtype, seed=seed, rest=float("nan"))
    Tq = sum(ql)
    Q = L.randn(Tq, Hq, D, seed=seed + 100, dtype=dtype)
    g = torch.Generator().manual_seed(seed)
    chosen = torch.full((Tq, Hk, count), -1, dtype=torch.int32)
    want, t = [], 0
    for s, (n, m) in enumerate(zip(ql, lens)):
        pages = -(-m // P)
        seen = torch.zeros((n, Hk, m), dtype=torch.bool)
        for i in range(n):
            for h in range(Hk):
                some = torch.randperm(pages, generator=g)[:count].sort().values if pick is None else pick(pages)
                chosen[t + i, h, :len(some)] = torch.as_tensor(some, dtype=torch.int32)
                for b in some.tolist() if torch.is_tensor(some) else some:
                    if 0 <= b < pages:
                        seen[i, h, b * P:(b + 1) * P] = True
            if causal:
                seen[i, :, max(0, m - n + i + 1):] = False
        want.append(U.masked(Q[t:t + n], c.K[s], c.V[s], seen.cuda(), 1 / math.sqrt(D) if scale is None else scale))
        t += n
    got = tdq.tdq_attention_selected(Q, c.k, c.v, chosen.cuda(), L.starts(ql), c.table, c.len, causal=causal, scale=scale,
                                     want_lse=True)
    L.check_attention(got, tuple(torch.cat(x) for x in zip(*want)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D", HEADS + [(40, 1, 128), (33, 1, 64)])
def test_chosen(Hq, Hk, D, dtype):
    for ql, lens, P, count in (([1], [1], 16, 1), ([1, 1], [500, 33], 16, 8), ([3, 0, 2], [200, 5, 31], 32, 4),
                               ([1], [3000], 16, 150), ([20], [333], 64, 3), ([1, 2], [4000, 0], 64, 40)):
        print(f"[chosen] {ql} {lens} P={P} count={count} {Hq}/{Hk} D={D} {dtype}", flush=True)
        for causal in (True, False):
            _chosen(ql, lens, P, Hq, Hk, D, dtype, count, causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D,T", [(32, 8, 128, 200), (16, 8, 64, 400), (12, 12, 32, 530), (16, 16, 8, 400), (8, 8, 256, 110),
                                       (20, 10, 96, 160), (18, 1, 184, 400), (6, 6, 200, 140), (16, 4, 64, 400), (32, 8, 128, 100),
                                       (8, 8, 256, 45), (8, 4, 32, 600), (16, 8, 72, 90)])
def test_lists_of_many_tokens(Hq, Hk, D, T, dtype):
    for ql, lens, P, count in (([T], [T + 50], 16, 5), ([T - 40, 1, 39], [T - 40, 700, 0], 32, 9), ([T // 2, T - T // 2], [4, 1300], 64, 3)):
        print(f"[chosen] {ql} {lens} P={P} count={count} {Hq}/{Hk} D={D} {dtype}", flush=True)
        for causal in (True, False):
            _chosen(ql, lens, P, Hq, Hk, D, dtype, count, causal)
    _chosen([T], [400], 16, Hq, Hk, D, dtype, 6, pick=lambda n: [5, -1, 0, 99999, n - 1, 3])


def test_chosen_in_any_order_and_none():
    _chosen([1, 4], [300, 100], 16, 4, 2, 64, torch.float16, 6, pick=lambda n: [5, -1, 0, 3])
    _chosen([1, 4], [300, 100], 16, 4, 2, 64, torch.float16, 6, pick=lambda n: [-1, -1, n - 1, 99999, -1, 2])
    _chosen([1, 4], [300, 100], 16, 4, 2, 64, torch.bfloat16, 6, pick=lambda n: [])
    _chosen([9], [4], 16, 4, 2, 64, torch.bfloat16, 2, pick=lambda n: [0])


def test_chosen_scales():
    for scale in (0.0, -0.3, 2.0):
        _chosen([2, 1], [300, 4000], 16, 4, 2, 64, torch.float16, 200, scale=scale)


def test_a_page_named_twice_counts_twice():
    c = U.Cache([48], 16, 1, 64, torch.bfloat16)
    Q = L.randn(1, 2, 64, seed=3, dtype=torch.bfloat16)
    got = tdq.tdq_attention_selected(Q, c.k, c.v, _i32([[[0, 2, 2]]]), L.starts([1]), c.table, c.len, want_lse=True)
    K, V = (torch.cat((x[0][:16], x[0][32:], x[0][32:])) for x in (c.K, c.V))
    L.check_attention(got, U.masked(Q, K, V, torch.ones((1, 1, 48), dtype=torch.bool, device="cuda"), 0.125))


def test_all_pages_chosen_is_the_whole_sequence():
    c = U.Cache([700, 90], 32, 2, 64, torch.float16)
    Q = L.randn(4, 8, 64, seed=3, dtype=torch.float16)
    every = torch.arange(22, dtype=torch.int32, device="cuda").expand(4, 2, 22).contiguous()
    want = U.sequences(Q, [3, 1], c, 0.125)
    L.check_attention(tdq.tdq_attention_selected(Q, c.k, c.v, every, L.starts([3, 1]), c.table, c.len, want_lse=True), want)


# ---- both --------------------------------------------------------------------------
def _calls(Q, k, v, cu, table, lens, chosen):
    return (lambda **kw: tdq.tdq_attention_paged(Q, k, v, cu, table, lens, want_lse=True, **kw),
            lambda **kw: tdq.tdq_attention_selected(Q, k, v, chosen, cu, table, lens, want_lse=True, **kw))


@pytest.mark.parametrize("ql", [[1, 2], [60, 50]])
def test_strides(ql):
    """Parts of a fused projection, heads outermost in the cache, an output with gaps, a table with gaps."""
    Hq, Hk, D, P = 4, 2, 64, 16
    c = U.Cache([300, 77], P, Hk, D, torch.bfloat16)
    T = sum(ql)
    qkv = L.randn(T, Hq + 2 * Hk, D, seed=1, dtype=torch.bfloat16)
    Q, cu = qkv[:, :Hq], L.starts(ql)
    chosen = torch.arange(4, dtype=torch.int32, device="cuda").expand(T, Hk, 4).contiguous()
    wide = torch.full((2, 40), 12345678, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    kh, vh = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (c.k, c.v))
    plain = _calls(Q.contiguous(), c.k, c.v, cu, c.table, c.len, chosen)
    other = _calls(Q, kh, vh, cu, wide[:, :c.table.shape[1]], c.len, chosen)
    for a, b in zip(plain, other):
        want = a()
        buf = torch.full((T, Hq + 3, D + 8), 55.0, dtype=torch.bfloat16, device="cuda")
        O, lse = b(out=buf[:, 1:1 + Hq, :D])
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
        assert bool((buf[:, 0] == 55).all()) and bool((buf[:, 1 + Hq:] == 55).all()) and bool((buf[..., D:] == 55).all())


def test_cache_beyond_32_bit_offsets():
    Hk, D, P, step = 2, 64, 16, 1 << 31
    c = U.Cache([40], P, Hk, D, torch.float16)
    room = torch.zeros((5 * step + P * Hk * D,), dtype=torch.float16, device="cuda")
    far = torch.as_strided(room, (6, P, Hk, D), (step, Hk * D, D, 1))
    chosen, cu = _i32([[[0, 1, 2]] * 2]), L.starts([1])
    Q = L.randn(1, 4, D, seed=9, dtype=torch.float16)
    want = [f() for f in _calls(Q, c.k, c.v, cu, c.table, c.len, chosen)]
    far.copy_(c.k)
    for f, w in zip(_calls(Q, far, c.v, cu, c.table, c.len, chosen), want):
        got = f()
        assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
    far.copy_(c.v)
    for f, w in zip(_calls(Q, c.k, far, cu, c.table, c.len, chosen), want):
        assert torch.equal(f()[0], w[0])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_nobody_sees_does_not_matter(bad):
    """Rows behind a sequence's last key, pages of others, pages that are not there."""
    for ql, lens in (([30, 1], [70, 90]), ([1, 1], [5, 3000]), ([200, 1], [333, 17])):
        got = []
        for rest in (0.0, bad):
            c = U.Cache(lens, 64, 2, 64, torch.float16, rest=rest)
            Q = L.randn(sum(ql), 4, 64, seed=1, dtype=torch.float16)
            chosen = torch.arange(6, dtype=torch.int32, device="cuda").expand(sum(ql), 2, 6).contiguous()
            got.append([x for f in _calls(Q, c.k, c.v, L.starts(ql), c.table, c.len, chosen) for x in f()])
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_values_that_are_not_finite_reach_who_sees_them():
    c = U.Cache([3000], 16, 1, 64, torch.bfloat16)
    Q = L.randn(1, 2, 64, seed=1, dtype=torch.bfloat16)
    chosen = torch.arange(188, dtype=torch.int32, device="cuda").view(1, 1, -1)
    c.k[c.lines[0][100], 3] = float("nan")
    for f in _calls(Q, c.k, c.v, L.starts([1]), c.table, c.len, chosen):
        O, lse = f()
        assert bool(torch.isnan(O).all()) and bool(torch.isnan(lse).all())
    c.k[c.lines[0][100], 3] = 0
    c.v[c.lines[0][50], 3, 0, 7] = float("inf")
    for f in _calls(Q, c.k, c.v, L.starts([1]), c.table, c.len, chosen):
        O, lse = f()
        assert bool((O[..., 7] == math.inf).all()) and int(torch.isfinite(O).sum()) == 2 * 63 and bool(torch.isfinite(lse).all())


def test_repeatable_and_in_any_stream():
    c = U.Cache([5000, 12, 800], 64, 2, 128, torch.bfloat16)
    Q = L.randn(3, 8, 128, seed=1, dtype=torch.bfloat16)
    chosen = torch.arange(60, dtype=torch.int32, device="cuda").expand(3, 2, 60).contiguous()
    calls = _calls(Q, c.k, c.v, L.starts([1, 1, 1]), c.table, c.len, chosen)
    want = [f() for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append([f() for f in calls])
        torch.cuda.synchronize()
        for g in got:
            for a, b in zip(g, want):
                assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
