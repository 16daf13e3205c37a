"""Attention over many keys of little weight each beside one that has nearly all of it."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("low,high", [(20.0, 26.0), (25.5, 29.0)])
@pytest.mark.parametrize("nq,Hq,n", [(1, 1, 30000), (2, 4, 30000), (1, 2, 300), (90, 1, 8000)])
def test_keys_far_below_the_largest(nq, Hq, n, low, high, dtype):
    """The first key has the largest score and values of zero, as a sink has; the others lie `low` to `high` octaves
    below it and give the whole output.

    Scores are exact: scale ln 2, one element of a key holds its octaves.  A probability is rounded to the type of V:
    relative to it, u, and for binary16 absolutely by half of its smallest number, 2^-25.  The largest probability is
    held at 2^7 at least, which makes that 2^-32 of the sum; twice as much is allowed, as for the ordinary cases."""
    D = 64
    g = L.gen(5)
    octaves = low + (high - low) * torch.rand((n,), generator=g, device="cuda")
    octaves = torch.round(octaves * 8) / 8                   # (8 bits: exact in both types)
    octaves[0] = 0.0
    Q = torch.zeros((nq, Hq, D), dtype=dtype, device="cuda")
    Q[..., 0] = 1.0
    K = torch.zeros((n, 1, D), dtype=dtype, device="cuda")
    K[:, 0, 0] = -octaves.to(dtype)
    assert torch.equal(K[:, 0, 0].float(), -octaves)
    V = (1.0 + 0.3 * torch.randn((n, 1, D), generator=g, device="cuda")).to(dtype)
    V[0] = 0.0
    O, lse = tdq.tdq_attention(Q, K, V, L.starts([nq]), L.starts([n]), scale=math.log(2.0), causal=False, want_lse=True)
    w = torch.exp2(-octaves.double())
    total = w.sum()
    want, size = (w @ V[:, 0].double()) / total, (w @ V[:, 0].double().abs()) / total
    u = L.UNIT[dtype]
    least = 2.0 ** -32 if dtype == torch.float16 else 0.0
    tol = u * want.abs() + (u + (n / 64 + 8) * 2.0 ** -23) * size + 2 * least * V[:, 0].double().abs().sum(dim=0)
    tol = tol + 2 * L.TINY[dtype]                            # the result's own smallest number
    bad = (O.double() - want).abs() / tol
    assert float(bad.max()) <= 1.0, float(bad.max())
    assert float((lse.double() - torch.log(total)).abs().max()) <= (n / 64 + 8) * 2.0 ** -23


def test_log_of_the_sum_where_all_scores_are_equal():
    """n equal scores: lse is their score and log n, in every way the keys are gone through."""
    for nq, n, Hq in ((1, 5000, 1), (1, 200, 2), (90, 300, 1), (1, 1, 1)):
        for dtype in (torch.float16, torch.bfloat16):
            Q = torch.full((nq, Hq, 32), 0.5, dtype=dtype, device="cuda")
            K = torch.full((n, 1, 32), 0.25, dtype=dtype, device="cuda")
            O, lse = tdq.tdq_attention(Q, K, K, L.starts([nq]), L.starts([n]), scale=1.0, causal=False, want_lse=True)
            want = 4.0 + math.log(n)
            assert float((lse.double() - want).abs().max()) <= (n / 64 + 8) * 2.0 ** -23 + 4 * 2.0 ** -24 * want
            assert float((O.double() - 0.25).abs().max()) <= 0.25 * (2 * L.UNIT[dtype] + (n / 64 + 8) * 2.0 ** -23)
