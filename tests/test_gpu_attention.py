"""Softmax attention over packed sequences, against 64 bits."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu


def _inputs(ql, kl, Hq, Hk, D, dtype, seed=0):
    Q = L.randn(sum(ql), Hq, D, seed=seed, dtype=dtype)
    K = L.randn(max(sum(kl), 0), Hk, D, seed=seed + 1, dtype=dtype)
    V = (L.randn(max(sum(kl), 0), Hk, D, seed=seed + 2) + 0.3).to(dtype)
    return Q, K, V


def _check(ql, kl, Hq, Hk, D, dtype, causal, scale=None, seed=0):
    Q, K, V = _inputs(ql, kl, Hq, Hk, D, dtype, seed)
    got = tdq.tdq_attention(Q, K, V, L.starts(ql), L.starts(kl), scale=scale, causal=causal, want_lse=True)
    L.check_attention(got, L.attention(Q, K, V, ql, kl, 1 / math.sqrt(D) if scale is None else scale, causal))


LENGTHS = [([1], [1]), ([5], [5]), ([64], [64]), ([65], [65]), ([33, 1, 200], [33, 1, 200]),
           ([0, 7, 0, 130, 0], [0, 7, 0, 130, 0]), ([3, 40, 1], [100, 41, 700]), ([129, 300], [129, 555])]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hk,D", [(1, 1, 64), (4, 2, 128), (6, 2, 32), (3, 1, 80), (8, 1, 96), (2, 2, 256),
                                     (5, 5, 8), (7, 1, 40), (2, 1, 200)])
def test_lengths(Hq, Hk, D, dtype, causal):
    for i, (ql, kl) in enumerate(LENGTHS):
        print(f"[attention] {ql} {kl} {Hq}/{Hk} D={D} {dtype} causal={causal}", flush=True)
        _check(ql, kl, Hq, Hk, D, dtype, causal, seed=i)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("ql,kl,Hq,Hk,D", [([1] * 5, [1, 63, 64, 65, 3001], 32, 8, 128), ([1], [9000], 8, 8, 64),
                                           ([1, 1, 0, 1], [0, 17, 5, 2000], 4, 1, 128), ([4, 2, 1], [4, 1000, 333], 16, 2, 64),
                                           ([1] * 130, list(range(130)), 2, 1, 32), ([1], [5000], 40, 1, 128),
                                           ([1, 1], [4097, 12], 6, 2, 256)])
def test_single_tokens(ql, kl, Hq, Hk, D, dtype):
    print(f"[attention] step {len(ql)} sequences {Hq}/{Hk} D={D} {dtype}", flush=True)
    for causal in (True, False):
        _check(ql, kl, Hq, Hk, D, dtype, causal, seed=3)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_prompts(dtype):
    _check([1000, 17, 2049], [1000, 17, 2049], 8, 2, 128, dtype, True)
    _check([700, 300], [1900, 301], 4, 4, 64, dtype, True)
    _check([512, 100], [77, 1500], 4, 2, 64, dtype, False)
    _check([1500], [1500], 12, 1, 64, dtype, True)


@pytest.mark.parametrize("causal", [False, True])
def test_queries_that_see_no_key(causal):
    """Fewer keys than queries under the causal rule: the first queries see none; sequences without keys."""
    _check([10, 70, 5], [4, 3, 0], 4, 2, 64, torch.float16, causal)
    _check([200], [130], 2, 1, 128, torch.bfloat16, causal)
    _check([1, 9], [0, 0], 2, 2, 64, torch.float16, causal)


def test_many_sequences():
    n = 5000
    ql = [(i * 7) % 4 for i in range(n)]
    kl = [(i * 5) % 9 for i in range(n)]
    Q, K, V = _inputs(ql, kl, 2, 1, 32, torch.float16)
    O, lse = tdq.tdq_attention(Q, K, V, L.starts(ql), L.starts(kl), causal=False, want_lse=True)
    pick = [0, 1, 2, 63, 64, 65, 2500, 4095, 4096, 4097, 4997, 4998, 4999]
    cq, ck = L.starts(ql).tolist(), L.starts(kl).tolist()
    for i in pick:
        a, b = slice(cq[i], cq[i + 1]), slice(ck[i], ck[i + 1])
        if ql[i]:
            want = L.attention(Q[a], K[b], V[b], [ql[i]], [kl[i]], 1 / math.sqrt(32), False)
            L.check_attention((O[a], lse[a]), want)


def test_large_and_growing_scores():
    """Scores of hundreds, the largest key last or first, so that the running maximum moves all the time or never."""
    n, D = 700, 64
    Q, K, V = _inputs([40], [n], 2, 1, D, torch.bfloat16)
    Q = Q.abs()
    up = torch.linspace(-3, 3, n, device="cuda")
    for ramp in (up, -up, up * 0):
        Kr = (ramp[:, None, None] * torch.ones((n, 1, D), device="cuda")).bfloat16()
        for scale in (1.0, 0.05):
            got = tdq.tdq_attention(Q, Kr, V, L.starts([40]), L.starts([n]), scale=scale, causal=True, want_lse=True)
            L.check_attention(got, L.attention(Q, Kr, V, [40], [n], scale, True))


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    _check([50, 1], [50, 400], 4, 2, 64, torch.float16, True, scale=scale)


def test_strides():
    """Parts of a fused projection, heads outermost, an output with gaps, one long step between tokens."""
    T, Hq, Hk, D = 150, 4, 2, 64
    qkv = L.randn(T, Hq + 2 * Hk, D, seed=1, dtype=torch.bfloat16)
    Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    cu = L.starts([100, 50])
    want = tdq.tdq_attention(Q.contiguous(), K.contiguous(), V.contiguous(), cu, cu, want_lse=True)
    buf = torch.full((T, Hq + 3, D + 8), 55.0, dtype=torch.bfloat16, device="cuda")
    O, lse = tdq.tdq_attention(Q, K, V, cu, cu, out=buf[:, 1:1 + Hq, :D], want_lse=True)
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    assert bool((buf[:, 0] == 55).all()) and bool((buf[:, 1 + Hq:] == 55).all()) and bool((buf[..., D:] == 55).all())
    Kh, Vh = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (K, V))
    O, lse = tdq.tdq_attention(Q, Kh, Vh, cu, cu, want_lse=True)
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])


def test_cache_beyond_32_bit_offsets():
    """Keys and values more than 2^32 elements from their tensor's start."""
    Hk, D, n = 2, 64, 600
    step = 8 * 1024 * 1024                                   # elements between tokens: 600 of them are 5 * 2^30
    room = torch.zeros(((n - 1) * step + Hk * D,), dtype=torch.float16, device="cuda")
    view = torch.as_strided(room, (n, Hk, D), (step, D, 1))
    _, K, V = _inputs([1], [n], Hk, Hk, D, torch.float16)
    Q = L.randn(3, 4, D, seed=9, dtype=torch.float16)
    cu_q, cu_k = L.starts([1, 2]), L.starts([n - 50, 50])
    want = tdq.tdq_attention(Q, K, V, cu_q, cu_k, want_lse=True)
    view.copy_(K)
    a = tdq.tdq_attention(Q, view, V, cu_q, cu_k, want_lse=True)
    assert torch.equal(a[0], want[0]) and torch.equal(a[1], want[1])
    view.copy_(V)
    b = tdq.tdq_attention(Q, K, view, cu_q, cu_k, want_lse=True)
    assert torch.equal(b[0], want[0])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_lies_outside_a_sequence_does_not_matter(bad):
    """NaN and infinities in the tokens between and after the sequences, and in another sequence."""
    D = 64
    ql, kl = [30, 20, 1], [70, 33, 90]
    Q, K, V = _inputs(ql, kl, 4, 2, D, torch.float16)
    want = tdq.tdq_attention(Q, K, V, L.starts(ql), L.starts(kl), want_lse=True)
    K2, V2 = K.clone(), V.clone()
    K2[70:103], V2[70:103] = bad, bad
    got = tdq.tdq_attention(Q, K2, V2, L.starts(ql), L.starts(kl), want_lse=True)
    for a, b in ((slice(0, 30), slice(0, 30)), (slice(50, 51), slice(50, 51))):
        assert torch.equal(got[0][a], want[0][b]) and torch.equal(got[1][a], want[1][b])
    cu_k = L.starts(kl)
    cu_k[3] -= 21                                            # the last sequence ends before the tensor does
    Q3 = Q[50:51]
    want = tdq.tdq_attention(Q3, K[103:172].contiguous(), V[103:172].contiguous(), L.starts([1]), L.starts([69]))
    K2, V2 = K.clone(), V.clone()
    K2[172:], V2[172:] = bad, bad
    cu_q = torch.tensor([0, 0, 0, 1], dtype=torch.int32, device="cuda")
    got = tdq.tdq_attention(Q3, K2, V2, cu_q, cu_k)
    assert torch.equal(got[0], want[0])


def test_offsets_outside_the_tensors_are_cut_off():
    D = 32
    Q, K, V = _inputs([20], [40], 2, 1, D, torch.float16)
    t = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    want = tdq.tdq_attention(Q, K, V, t(0, 20), t(0, 40), causal=False)[0]
    got = tdq.tdq_attention(Q, K, V, t(-5, 900), t(-1, 4000), causal=False)[0]
    assert torch.equal(got, want)
    out = torch.full((20, 2, D), 9.0, dtype=torch.float16, device="cuda")
    tdq.tdq_attention(Q, K, V, t(3, 8), t(0, 40), causal=False, out=out)
    assert torch.equal(out[3:8], want[3:8]) and bool((out[:3] == 9).all()) and bool((out[8:] == 9).all())


def test_no_keys_at_all():
    Q = L.randn(5, 2, 64, dtype=torch.float16)
    K = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    O, lse = tdq.tdq_attention(Q, K, K, L.starts([2, 3]), L.starts([0, 0]), want_lse=True)
    assert bool((O == 0).all()) and bool((lse == -math.inf).all())


def test_repeats_and_streams():
    ql, kl = [1, 1, 1], [3000, 10, 700]
    Q, K, V = _inputs(ql, kl, 8, 2, 128, torch.bfloat16)
    cu_q, cu_k = L.starts(ql), L.starts(kl)
    want = tdq.tdq_attention(Q, K, V, cu_q, cu_k, want_lse=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [tdq.tdq_attention(Q, K, V, cu_q, cu_k, want_lse=True) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(s)
    for O, lse in got:
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("ql,kl,Hq,Hk,D", [([130], [130], 2, 1, 64), ([70, 40], [200, 41], 4, 4, 128), ([7], [300], 4, 1, 128),
                                           ([4, 3], [40, 1000], 8, 2, 32), ([90], [90], 1, 1, 200)])
def test_keys_behind_the_causal_edge_may_be_anything(ql, kl, Hq, Hk, D, bad, dtype):
    """The last queries of a sequence see its last keys, which are NaN (or give NaN scores): the queries before them
    stay as they are, bit for bit."""
    Q, K, V = _inputs(ql, kl, Hq, Hk, D, dtype)
    cu_q, cu_k = L.starts(ql), L.starts(kl)
    print(f"[attention] {bad} behind the edge {ql} {kl} D={D} {dtype}", flush=True)
    want = tdq.tdq_attention(Q, K, V, cu_q, cu_k, want_lse=True)
    K2, touched = K.clone(), torch.zeros(Q.shape[0], dtype=torch.bool, device="cuda")
    for nq, q1, k1 in zip(ql, cu_q.tolist()[1:], cu_k.tolist()[1:]):
        late = nq // 2
        K2[k1 - late:k1, :, 0] = bad
        K2[k1 - late:k1, :, 1] = -bad
        touched[q1 - late:q1] = True
    Q2 = Q.clone()
    Q2[touched] = Q2[touched].abs()                          # (infinities of both signs: NaN)
    O, lse = tdq.tdq_attention(Q2, K2, V, cu_q, cu_k, want_lse=True)
    assert torch.equal(O[~touched], want[0][~touched]) and torch.equal(lse[~touched], want[1][~touched])
    assert bool(O[touched].float().isnan().all())


@pytest.mark.parametrize("nq", [1, 3, 40])
def test_cache_with_room(nq):
    """Sequences in equal rooms of a cache, of which the first few keys are used: the same as packed."""
    S, room, Hq, Hk, D = 5, 700, 8, 2, 64
    used = [700, 0, 1, 333, 64]
    Q, K, V = _inputs([nq] * S, [room] * S, Hq, Hk, D, torch.bfloat16)
    cu_q, cu_k = L.starts([nq] * S), L.starts([room] * S)
    keep = torch.cat([torch.arange(s * room, s * room + n, device="cuda") for s, n in enumerate(used)])
    want = L.attention(Q, K[keep], V[keep], [nq] * S, used, D ** -0.5, True)
    rest = torch.ones(S * room, dtype=torch.bool, device="cuda")
    rest[keep] = False
    K[rest], V[rest] = float("nan"), float("inf")
    n = torch.tensor(used, dtype=torch.int32, device="cuda")
    L.check_attention(tdq.tdq_attention(Q, K, V, cu_q, cu_k, len_k=n, want_lse=True), want)
    more = n + 10000                                         # more than there is room for: all of it; fewer than none: none
    a = tdq.tdq_attention(Q, K, V, cu_q, cu_k, len_k=more)[0]
    b = tdq.tdq_attention(Q, K, V, cu_q, cu_k)[0]
    assert torch.equal(a.isnan(), b.isnan())
    assert bool((tdq.tdq_attention(Q, K, V, cu_q, cu_k, len_k=-n - 1)[0] == 0).all())
