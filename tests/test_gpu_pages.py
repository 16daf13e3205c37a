"""A cache in pages: writing to it, the bounds of its pages and the choice of pages, against 64 bits."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L
import pages_util as U

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _places(ql, lens, table, P, n_pages, first=0):
    """(token, page, row, key) of the tokens that have a place, from the definition."""
    out, t = [], first
    for s, (n, m) in enumerate(zip(ql, lens)):
        for i in range(n):
            j = m - n + i
            if 0 <= j < table.shape[1] * P and 0 <= int(table[s, j // P]) < n_pages:
                out.append((t + i, int(table[s, j // P]), j % P, j))
        t += n
    return out


def _append(ql, lens, P, Hq, Hk, D, R, axes, inter, dtype, norm=True, table=None, first=0, behind=0, fused=True, seed=0,
            pos=None, own_place=False, outermost=False):
    T, Pn = first + sum(ql) + behind, R // 2
    n_pages = 3 + sum(-(-m // P) for m in lens)
    if table is None:
        ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        cols = max(1, max(-(-m // P) for m in lens))
        table = _i32([[ids.pop() if b < -(-m // P) else -1 for b in range(cols)] for m in lens])
    qkv = L.randn(T, Hq + 2 * Hk, D, seed=seed + 1, dtype=dtype)
    Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    if not fused:
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
    shape = (n_pages, Hk, P, D) if outermost else (n_pages, P, Hk, D)
    kc, vc = L.randn(*shape, seed=seed + 2, dtype=dtype), L.randn(*shape, seed=seed + 3, dtype=dtype)
    if outermost:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    k0, v0 = kc.clone(), vc.clone()
    wq, wk = (1 + 0.2 * L.randn(D, seed=s) for s in (1, 2)) if norm else (None, None)
    freq = (10000.0 ** (-torch.arange(Pn, device="cuda").double() / max(Pn, 1))).float() if Pn else None
    axis = (torch.arange(Pn, device="cuda") % axes).to(torch.int32) if axes > 1 else None
    if pos is None and not own_place:
        pos = torch.randint(0, 4000, (axes, T), generator=L.gen(3), device="cuda").to(torch.int32)
    cu = first + L.starts(ql)
    out = torch.full((T, Hq, D), 7.0, dtype=dtype, device="cuda")
    got = tdq.tdq_cache_append(Q if Hq else None, K, V, kc, vc, cu, table, _i32(lens), freq, pos=pos, q_weight=wq,
                               k_weight=wk, axis=axis, interleaved=inter, out=out if Hq else None)
    assert got is (out if Hq else None)
    places = _places(ql, lens, table.cpu(), P, n_pages, first)
    if pos is None:
        pos = torch.zeros((1, T), dtype=torch.int32)
        t = first
        for n, m in zip(ql, lens):
            pos[0, t:t + n] = torch.arange(m - n, m)
            t += n
        pos = pos.cuda()
    # the arithmetic of the head norm: about a dozen roundings of numbers no larger than a pair's, then the result's
    def close(y, x, w):
        want = L.norm_rotate(x, w, 1e-6, pos, freq, axis, inter)
        tol = 24 * 2.0 ** -24 * want.abs().amax(dim=-1, keepdim=True) + L.UNIT[dtype] * want.abs() + L.TINY[dtype]
        bad = ((y.double() - want).abs() / tol).masked_fill(y.double() == want, 0)
        return float(bad[first:T - behind].max()) <= 1.0 if T > first + behind else True
    if Hq:
        assert close(out, Q, wq)
        assert bool((out[:first] == 7).all()) and bool((out[T - behind:] == 7).all())
    written = torch.zeros((n_pages, P), dtype=torch.bool, device="cuda")
    if places:
        t, page, row, _ = (torch.tensor(x, device="cuda") for x in zip(*places))
        assert torch.equal(vc[page, row], V[t])
        full = K.clone()
        full.zero_()
        want = L.norm_rotate(K, wk, 1e-6, pos, freq, axis, inter)[t]
        tol = 24 * 2.0 ** -24 * want.abs().amax(dim=-1, keepdim=True) + L.UNIT[dtype] * want.abs() + L.TINY[dtype]
        y = kc[page, row].double()
        assert float(((y - want).abs() / tol).masked_fill(y == want, 0).max()) <= 1.0
        written[page, row] = True
    assert torch.equal(kc[~written], k0[~written]) and torch.equal(vc[~written], v0[~written])
    return len(places)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("Hq,Hk,D,R", [(1, 1, 8, 8), (32, 8, 128, 128), (6, 2, 80, 80), (4, 4, 96, 48), (3, 1, 256, 256),
                                       (2, 2, 40, 16), (7, 7, 72, 8), (2, 1, 248, 0), (0, 3, 64, 64)])
def test_append(Hq, Hk, D, R, inter, dtype):
    for ql, lens, P in (([1], [1], 16), ([1, 1, 1], [17, 1, 64], 16), ([5, 0, 33], [40, 9, 33], 32), ([70, 3], [70, 131], 64)):
        print(f"[append] {ql} {lens} P={P} {Hq}/{Hk} D={D} R={R} {inter} {dtype}", flush=True)
        assert _append(ql, lens, P, Hq, Hk, D, R, 1, inter, dtype) == sum(ql)


@pytest.mark.parametrize("dtype", TYPES)
def test_append_positions_axes_and_layouts(dtype):
    _append([40, 1], [50, 300], 16, 4, 2, 64, 64, 1, False, dtype, own_place=True)
    _append([40, 1], [50, 300], 16, 4, 2, 64, 32, 1, True, dtype, own_place=True, norm=False)
    _append([40, 1], [50, 300], 128, 4, 2, 96, 96, 2, False, dtype, fused=False)
    _append([40, 1], [50, 300], 1024, 4, 2, 96, 96, 3, True, dtype, outermost=True)
    _append([3000, 1, 2000], [3000, 7, 2500], 16, 2, 2, 32, 32, 1, False, dtype)   # several tokens a workgroup


def test_append_where_there_is_no_place():
    """More tokens than keys, more keys than the line has room for, pages that are not there, tokens of no sequence."""
    d = torch.float16
    assert _append([10, 4], [4, 6], 16, 2, 1, 64, 64, 1, False, d) == 8
    t = _i32([[0, 1], [2, 3]])
    assert _append([20, 3], [40, 33], 16, 2, 1, 64, 64, 1, False, d, table=t) == 12 + 2
    t = _i32([[0, -1], [99, 3]])
    assert _append([20, 20], [20, 20], 16, 2, 1, 64, 64, 1, False, d, table=t) == 16 + 4
    assert _append([5, 6], [5, 6], 16, 2, 1, 64, 64, 1, False, d, first=3, behind=9) == 11
    assert _append([5], [-3], 16, 2, 1, 64, 64, 1, False, d, table=_i32([[0]])) == 0
    assert _append([0, 0], [3, 0], 16, 2, 1, 64, 64, 1, False, d, behind=4) == 0


def test_append_in_place_equals_the_head_norm():
    """The same bits as tdq_norm_rotate and a copy."""
    T, Hq, Hk, D = 77, 8, 2, 128
    qkv = L.randn(T, Hq + 2 * Hk, D, dtype=torch.bfloat16)
    freq = (10000.0 ** (-torch.arange(D // 2, device="cuda").double() / (D // 2))).float()
    w = 1 + 0.1 * L.randn(D, seed=4)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    want = tdq.tdq_norm_rotate(Q, K, pos, freq, q_weight=w, k_weight=w)
    kc, vc = (torch.zeros((5, 16, Hk, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tdq.tdq_cache_append(Q, K, V, kc, vc, L.starts([T]), _i32([[4, 2, 0, 1, 3]]), _i32([T]), freq, q_weight=w,
                         k_weight=w, out=Q)
    assert torch.equal(Q, want[0])
    assert torch.equal(kc[[4, 2, 0, 1, 3]].flatten(0, 1)[:T], want[1])
    assert torch.equal(vc[[4, 2, 0, 1, 3]].flatten(0, 1)[:T], V)


def test_append_beyond_32_bit_offsets():
    """Pages more than 2^32 elements from their tensor's start."""
    Hk, D, P, step = 2, 64, 16, 1 << 31
    room = torch.zeros((2 * step + P * Hk * D,), dtype=torch.float16, device="cuda")
    kc = torch.as_strided(room, (3, P, Hk, D), (step, Hk * D, D, 1))
    vc = torch.zeros((3, P, Hk, D), dtype=torch.float16, device="cuda")
    K, V = L.randn(40, Hk, D, seed=1, dtype=torch.float16), L.randn(40, Hk, D, seed=2, dtype=torch.float16)
    t = _i32([[2, 0, 1]])
    tdq.tdq_cache_append(None, K, V, kc, vc, L.starts([40]), t, _i32([40]))
    assert torch.equal(kc[[2, 0, 1]].flatten(0, 1)[:40], K) and torch.equal(vc[[2, 0, 1]].flatten(0, 1)[:40], V)
    lo, hi = tdq.tdq_page_bounds(kc, t, _i32([40]))
    assert torch.equal(lo[2], K[:16].amin(dim=0)) and torch.equal(hi[1], K[32:].amax(dim=0))


# ---- bounds ------------------------------------------------------------------------
def _bounds(cache, ql, untouched):
    """The bounds of the pages that the last ql[s] keys lie in (ql None: of all), the others `untouched`."""
    lo, hi = untouched[0].clone(), untouched[1].clone()
    for s, (line, m) in enumerate(zip(cache.lines, cache.lengths)):
        for b, page in enumerate(line):
            if ql is None or (ql[s] > 0 and (b + 1) * cache.P > m - ql[s]):
                k = cache.K[s][b * cache.P:(b + 1) * cache.P]
                lo[page], hi[page] = k.amin(dim=0), k.amax(dim=0)
    return lo, hi


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hk,D,P", [(1, 8, 16), (8, 128, 64), (2, 64, 16), (3, 80, 32), (1, 256, 128), (5, 96, 1024), (4, 32, 16)])
def test_bounds(Hk, D, P, dtype):
    for lens, ql in (([1], [1]), ([P], [1]), ([P + 1], [1]), ([0, 3 * P + 5, 7], [0, 2 * P, 7]), ([5 * P - 1, 40], [0, 50]),
                     ([2 * P, P - 1, P + 3], [P + 1, 1, 4]), ([1] * 70, [i % 2 for i in range(70)])):
        c = U.Cache(lens, P, Hk, D, dtype, seed=len(lens), rest=1000.0)
        old = tuple(L.randn(c.k.shape[0], Hk, D, seed=s, dtype=dtype) for s in (8, 9))
        for q in (None, ql):
            out = tuple(x.clone() for x in old)
            got = tdq.tdq_page_bounds(c.k, c.table, c.len, cu_q=None if q is None else L.starts(q),
                                      Tq=None if q is None else sum(q), out=out)
            assert got[0] is out[0]
            want = _bounds(c, q, old)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (lens, q)


def test_bounds_of_strange_pages():
    """NaN is kept, infinities are values, pages that are not there and lines without room are passed over."""
    c = U.Cache([40, 20], 16, 2, 64, torch.bfloat16)
    c.k[c.lines[0][1], 3, 1, 5], c.k[c.lines[0][0], 15, 0, 7] = float("nan"), float("inf")
    c.k[c.lines[1][0], 0, 0, 9] = -float("inf")
    lo, hi = tdq.tdq_page_bounds(c.k, c.table, c.len)
    assert torch.isnan(lo[c.lines[0][1], 1, 5]) and torch.isnan(hi[c.lines[0][1], 1, 5])
    assert int(torch.isnan(lo).sum()) == 1 and int(torch.isnan(hi).sum()) == 1
    assert float(hi[c.lines[0][0], 0, 7]) == math.inf and float(lo[c.lines[1][0], 0, 9]) == -math.inf
    t = c.table.clone()
    t[0, 0], t[1, 1] = 1 << 30, -5
    lo, hi = tdq.tdq_page_bounds(c.k, t, _i32([4000, 20]))     # (more keys than the line has room for)
    for page, there in ((c.lines[0][0], False), (c.lines[0][2], True), (c.lines[1][0], True), (c.lines[1][1], False)):
        assert bool((hi[page] > 0).any()) is there


def test_bounds_of_a_cache_with_heads_outermost_and_odd_strides():
    c = U.Cache([100, 33], 32, 3, 40, torch.float16)
    k = torch.zeros((c.k.shape[0], 3, 32, 43), dtype=torch.float16, device="cuda")[..., 1:41].transpose(1, 2)
    k.copy_(c.k)
    lo, hi = tdq.tdq_page_bounds(k, c.table, c.len)
    want = tdq.tdq_page_bounds(c.k, c.table, c.len)
    assert torch.equal(lo, want[0]) and torch.equal(hi, want[1])


# ---- choice ------------------------------------------------------------------------
def _choice(Q, lo, hi, ql, lens, table, P, count, first, last, causal):
    """chosen[Tq, Hk, count] from the definition: sums in 64 bits, rounded to 32, lists sorted by the host."""
    Hq, Hk, g = Q.shape[1], lo.shape[1], Q.shape[1] // lo.shape[1]
    out, t = [], 0
    for s, (n, m) in enumerate(zip(ql, lens)):
        m = max(0, min(m, table.shape[1] * P))
        pages = -(-m // P)
        ids = table[s, :pages].long()
        there = ((ids >= 0) & (ids < lo.shape[0])).tolist()
        at = ids.clamp(0, lo.shape[0] - 1)
        for i in range(n):
            sees = m - n + i + 1 if causal else m
            seen = max(0, -(-sees // P))
            row = []
            for h in range(Hk):
                q = Q[t + i, h * g:(h + 1) * g].double()
                z = (q.clamp(min=0)[:, None] * hi[at, h].double()).sum(-1) + (q.clamp(max=0)[:, None] * lo[at, h].double()).sum(-1)
                z = z.float().amax(dim=0)[:seen].tolist() if pages else []
                always = [b < first or b >= seen - last for b in range(seen)]
                row.append(U.best(z, there, always, count))
            out.append(row)
        t += n
    return torch.tensor(out, dtype=torch.int32, device="cuda").view(-1, Hk, count)


def _check_choice(ql, lens, P, Hq, Hk, D, dtype, count, first=1, last=1, causal=True, seed=0, change=None):
    c = U.Cache(lens, P, Hk, 8, dtype, seed=seed)
    n = c.k.shape[0]
    mid, wide = L.randn(n, Hk, D, seed=seed + 1), 1 + L.randn(n, Hk, D, seed=seed + 2).abs()
    lo, hi = (mid - wide).to(dtype), (mid + wide).to(dtype)
    Q, table = L.randn(sum(ql), Hq, D, seed=seed + 3, dtype=dtype), c.table
    if change:
        Q, lo, hi, table = change(Q, lo, hi, table)
    got = tdq.tdq_select_pages(Q, lo, hi, L.starts(ql), table, c.len, P, count, first=first, last=last, causal=causal)
    want = _choice(Q, lo, hi, ql, lens, table, P, count, first, last, causal)
    assert torch.equal(got, want), (got != want).nonzero()[:5].tolist()
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D", [(1, 1, 8), (32, 8, 128), (6, 2, 64), (3, 1, 80), (8, 1, 96), (4, 4, 256), (5, 1, 40)])
def test_choice(Hq, Hk, D, dtype):
    for ql, lens, P, count in (([1], [1], 16, 1), ([1, 1], [500, 33], 16, 8), ([3, 0, 2], [200, 5, 31], 32, 4),
                               ([1], [3000], 16, 128), ([2], [130 * 16], 16, 40)):
        print(f"[choice] {ql} {lens} P={P} count={count} {Hq}/{Hk} D={D} {dtype}", flush=True)
        for first, last in ((1, 1), (0, 0), (0, 1)):
            if first + last <= count:
                _check_choice(ql, lens, P, Hq, Hk, D, dtype, count, first, last)
    _check_choice([4, 1], [90, 3], 16, Hq, Hk, D, dtype, 3, causal=False)
    _check_choice([9, 3], [5, 0], 16, Hq, Hk, D, dtype, 2)             # queries that see nothing


def test_choice_of_many_pages():
    """More pages than stay in registers, nearly all of them, and two thirds."""
    _check_choice([1, 2], [16 * 2050 + 3, 16 * 5000], 16, 2, 1, 16, torch.float16, 40, 2, 3)
    _check_choice([1], [16 * 4000], 16, 1, 1, 16, torch.bfloat16, 3999)
    _check_choice([1], [16 * 4000 - 5], 16, 1, 1, 16, torch.bfloat16, 2700, 0, 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D,T", [(8, 2, 64, 1030), (4, 4, 32, 2050), (12, 4, 128, 520), (16, 8, 80, 530), (10, 1, 256, 2060),
                                       (64, 64, 8, 260)])
def test_choice_of_many_tokens(Hq, Hk, D, T, dtype):
    """Tokens of a sequence together: runs that end inside a workgroup's tokens, queries that see few pages or none."""
    for ql, lens, P, count, causal in (([T], [T], 32, 4, True), ([T - 203, 3, 200], [T + 300, 5, 150], 64, 6, True),
                                       ([T - 77, 0, 77], [500, 100, 16 * 200], 16, 9, False)):
        print(f"[choice] {ql} {lens} P={P} count={count} {Hq}/{Hk} D={D} {dtype}", flush=True)
        _check_choice(ql, lens, P, Hq, Hk, D, dtype, count, causal=causal)


def test_choice_of_many_tokens_and_pages():
    """As many pages as fit, nearly all of them, one more than fit; scores that tie, strange ones, no sequence."""
    def few(Q, lo, hi, table):
        return Q.sign(), torch.full_like(lo, -1), (torch.arange(hi.shape[0], device="cuda") % 3)[:, None, None].to(hi.dtype).expand_as(hi).contiguous(), table

    def strange(Q, lo, hi, table):
        hi[table[0, 7], 0, 3], hi[table[0, 9], 0, 2], lo[table[0, 11]] = float("nan"), float("inf"), -float("inf")
        table = table.clone()
        table[0, 0], table[0, 5], table[0, 40] = -1, 1 << 30, -7
        return Q, lo, hi, table

    T = 260
    for pages in (1024, 1025):
        _check_choice([T], [16 * pages - 3], 16, 8, 8, 16, torch.float16, 40, 2, 3)
    _check_choice([T], [16 * 1000], 16, 32, 8, 16, torch.bfloat16, 990)
    _check_choice([T], [16 * 300], 16, 32, 8, 32, torch.float16, 50, change=few)
    for count in (1, 3, 60, 200):
        _check_choice([T], [16 * 100], 16, 32, 8, 32, torch.float16, count, min(1, count - 1), 0, change=strange)
    _check_choice([T], [16 * 100], 16, 32, 8, 32, torch.bfloat16, 4, change=lambda Q, lo, hi, t: (Q, lo, hi, t * 0 - 1))
    c = U.Cache([700], 16, 1, 8, torch.float16)
    n = c.k.shape[0]
    lo, hi = L.randn(n, 8, 32, seed=1, dtype=torch.float16), L.randn(n, 8, 32, seed=2, dtype=torch.float16)
    Q = L.randn(300, 32, 32, dtype=torch.float16)
    out = torch.full((300, 8, 5), 77, dtype=torch.int32, device="cuda")
    tdq.tdq_select_pages(Q, lo, hi, _i32([6, 280]), c.table, c.len, 16, 5, out=out)
    assert bool((out[:6] == 77).all()) and bool((out[280:] == 77).all())
    assert torch.equal(out[6:280], _choice(Q[6:280], lo, hi, [274], [700], c.table, 16, 5, 1, 1, True))


def test_choice_where_scores_tie():
    """Few different scores: the lower page is better.  All the same, and zeros of both signs."""
    def few(Q, lo, hi, table):
        return Q.sign(), torch.full_like(lo, -1), (torch.arange(hi.shape[0], device="cuda") % 3)[:, None, None].to(hi.dtype).expand_as(hi).contiguous(), table

    def same(Q, lo, hi, table):
        return Q, torch.zeros_like(lo), torch.zeros_like(hi), table

    def signs(Q, lo, hi, table):
        z = torch.where(torch.arange(hi.shape[0], device="cuda") % 2 == 0, 0.0, -0.0)[:, None, None].expand_as(hi)
        return Q, z.to(lo.dtype).contiguous(), z.to(hi.dtype).contiguous(), table

    for change in (few, same, signs):
        _check_choice([2], [16 * 700], 16, 2, 1, 64, torch.float16, 50, change=change)
        _check_choice([1], [16 * 3000], 16, 2, 1, 32, torch.bfloat16, 50, 0, 0, change=change)


def test_choice_with_strange_scores():
    """NaN counts as largest, infinities as they are, pages that are not there are not taken (not even always)."""
    def strange(Q, lo, hi, table):
        hi[table[0, 7], 0, 3], hi[table[0, 9], 0, 2], lo[table[0, 11]] = float("nan"), float("inf"), -float("inf")
        hi[table[0, 13]] = -float("inf")
        table = table.clone()
        table[0, 0], table[0, 5], table[0, 40] = -1, 1 << 30, -7
        return Q, lo, hi, table

    for count in (1, 2, 3, 10, 30, 60):
        _check_choice([1, 3], [16 * 41, 300], 16, 4, 2, 64, torch.float16, count, min(1, count - 1), 1, change=strange)
    _check_choice([1], [100], 16, 2, 2, 64, torch.bfloat16, 4, change=lambda Q, lo, hi, t: (Q, lo, hi, t * 0 - 1))


def test_choice_leaves_tokens_of_no_sequence_alone():
    c = U.Cache([100], 16, 1, 8, torch.float16)
    lo, hi = L.randn(10, 1, 32, seed=1, dtype=torch.float16), L.randn(10, 1, 32, seed=2, dtype=torch.float16)
    Q = L.randn(9, 2, 32, dtype=torch.float16)
    out = torch.full((9, 1, 5), 77, dtype=torch.int32, device="cuda")
    tdq.tdq_select_pages(Q, lo, hi, _i32([2, 6]), c.table, c.len, 16, 5, out=out)
    assert bool((out[:2] == 77).all()) and bool((out[6:] == 77).all())
    assert torch.equal(out[2:6], _choice(Q[2:6], lo, hi, [4], [100], c.table, 16, 5, 1, 1, True))


def test_choice_bounds_every_product():
    """No key has a larger product with a query than its page's score says."""
    c = U.Cache([300], 16, 1, 64, torch.bfloat16)
    lo, hi = tdq.tdq_page_bounds(c.k, c.table, c.len)
    Q = L.randn(1, 4, 64, seed=3, dtype=torch.bfloat16)
    got = tdq.tdq_select_pages(Q, lo, hi, L.starts([1]), c.table, c.len, 16, 6, first=0, last=0)[0, 0].tolist()
    q, line = Q[0].double(), c.table[0].long()
    score = (q.clamp(min=0) @ hi[line, 0].double().t().contiguous() + q.clamp(max=0) @ lo[line, 0].double().t().contiguous()).amax(dim=0)
    dots = (q @ c.K[0][:, 0].double().t().contiguous()).amax(dim=0)
    assert all(float(dots[16 * b:16 * b + 16].max()) <= float(score[b]) for b in range(19))
    assert got == sorted(score.argsort(descending=True)[:6].tolist())
