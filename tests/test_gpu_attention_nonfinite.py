"""Attention where queries, keys or values are not finite: NaN reaches every row that sees it, whichever way the keys
are shared out, and no other."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu

# (queries, keys, query heads, key heads, D): the keys of a sequence cut into parts that a second launch joins, into
# wavefronts of one workgroup, and rows that go through all keys
SPLIT = ([1, 1, 2], [3000, 700, 2500], 8, 2, 128)
WAVES = ([1, 3, 2], [400, 33, 150], 8, 2, 64)
ROWS = ([70, 40], [300, 200], 4, 2, 64)
WAYS = [SPLIT, WAVES, ROWS]


def _inputs(way, dtype, seed=0):
    ql, kl, Hq, Hk, D = way
    Q, K, V = (L.randn(n, h, D, seed=seed + i, dtype=dtype) for i, (n, h) in
               enumerate([(sum(ql), Hq), (sum(kl), Hk), (sum(kl), Hk)]))
    cut = tdq.tdq_attention_workspace_bytes(sum(ql), sum(kl), len(ql), Hq, Hk, D) > 0
    assert cut == (way is SPLIT)
    return Q, K, V, L.starts(ql), L.starts(kl)


def _run(Q, K, V, cu_q, cu_k, causal=False, **kw):
    return tdq.tdq_attention(Q, K, V, cu_q, cu_k, causal=causal, want_lse=True, **kw)


def _only(got, want, hit):
    """NaN in the rows `hit` [Tq, Hq], in O and lse; the others as without, bit for bit."""
    O, lse = got
    assert bool(O[hit].float().isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(O[~hit], want[0][~hit]) and torch.equal(lse[~hit], want[1][~hit])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("way", WAYS)
def test_a_nan_query(way, dtype):
    Q, K, V, cu_q, cu_k = _inputs(way, dtype)
    want = _run(Q, K, V, cu_q, cu_k)
    hit = torch.zeros(Q.shape[:2], dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[Q.shape[0] - 1] = True
    Q[0, 1, 3], Q[Q.shape[0] - 1] = float("nan"), float("nan")
    _only(_run(Q, K, V, cu_q, cu_k), want, hit)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("part", ["first half", "second half", "a tile", "whole parts", "all"])
def test_runs_of_nan_keys(way, part, dtype):
    """Of one key head of the first sequence.  (Whole parts: tiles 12 to 35 of 32 keys, where a split has 12.)"""
    Q, K, V, cu_q, cu_k = _inputs(way, dtype)
    ql, kl, Hq, Hk, _ = way
    want = _run(Q, K, V, cu_q, cu_k)
    n = kl[0]
    a, b = {"first half": (0, n // 2), "second half": (n // 2, n), "a tile": (32, 64),
            "whole parts": (384, 1152), "all": (0, n)}[part]
    b = min(b, n)
    a = min(a, b - 1)
    K[a:b, 1] = float("nan")
    hit = torch.zeros(Q.shape[:2], dtype=torch.bool, device="cuda")
    hit[:ql[0], Hq // Hk:2 * (Hq // Hk)] = True
    _only(_run(Q, K, V, cu_q, cu_k), want, hit)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("way", WAYS)
def test_infinite_scores(way, dtype):
    """A score of -inf is a weight of 0, as if the key were not there; one of +inf leaves no quotient: NaN."""
    ql, kl, Hq, Hk, D = way
    Q, K, V, cu_q, cu_k = _inputs(way, dtype)
    Q = Q.abs() + 0.25
    K[5] = 0.0
    K2 = K.clone()
    K2[5, :, 7] = -math.inf
    keep = torch.arange(K.shape[0], device="cuda") != 5
    want = L.attention(Q, K[keep], V[keep], ql, [kl[0] - 1] + kl[1:], D ** -0.5, False)
    L.check_attention(_run(Q, K2, V, cu_q, cu_k), want)
    K2[5, :, 7] = math.inf
    O, _ = _run(Q, K2, V, cu_q, cu_k)
    assert bool(O[:ql[0]].float().isnan().all()) and bool(O[ql[0]:].isfinite().all())


@pytest.mark.parametrize("way", [([4, 1], [2, 3000], 8, 2, 128), ([10, 3], [4, 0], 4, 2, 64), ([70, 5], [40, 0], 4, 2, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_without_a_key_among_values_that_are_not_finite(way, bad):
    """The first queries of a sequence with fewer keys than queries see none: zeros, and -inf, whatever the values."""
    ql, kl, Hq, Hk, D = way
    Q, K, V = (L.randn(n, h, D, seed=i, dtype=torch.float16) for i, (n, h) in
               enumerate([(sum(ql), Hq), (sum(kl), Hk), (sum(kl), Hk)]))
    V[:kl[0]] = bad
    O, lse = _run(Q, K, V, L.starts(ql), L.starts(kl), causal=True)
    none = ql[0] - kl[0]
    assert bool((O[:none] == 0).all()) and bool((lse[:none] == -math.inf).all())
    assert not bool(O[none:ql[0]].isfinite().any()) and bool(lse[none:ql[0]].isfinite().all())
    rest = O[ql[0]:]
    assert bool(rest.isfinite().all()) and (kl[1] > 0 or bool((rest == 0).all()))


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("part", ["first half", "second half", "whole parts"])
def test_values_of_no_weight_still_count(way, bad, part):
    """Keys whose scores are 2000 below the others' and whose values are not finite: 0 * NaN is NaN."""
    ql, kl, Hq, Hk, D = way
    Q, K, V, cu_q, cu_k = _inputs(way, torch.bfloat16)
    Q[:], K[:] = 1.0, 0.0
    n = kl[0]
    half = {"first half": slice(0, n // 2), "second half": slice(n // 2, n),
            "whole parts": slice(min(384, n // 3), min(1152, n - 1))}[part]
    K[half, :, 0] = -2000.0
    want = _run(Q, K, V, cu_q, cu_k, scale=1.0)
    V[half] = bad
    O, lse = _run(Q, K, V, cu_q, cu_k, scale=1.0)
    assert bool(O[:ql[0]].float().isnan().all()) and torch.equal(lse, want[1])
    assert torch.equal(O[ql[0]:], want[0][ql[0]:])
