"""The choice of pages where some scores are the lowest that there are, and as many pages are there as are wanted."""
import math

import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L
from test_gpu_pages import _choice

pytestmark = pytest.mark.gpu


def _lowest(low, places, missing, value):
    """Pages `places` of the first line score `value` for every query (the first channel of all queries is 1), those of
    `missing` are not there; no score is NaN."""
    def change(Q, lo, hi, table):
        Q[..., 0] = 1
        at = table[0, places].long()
        lo[at], hi[at] = 0, 0
        hi[at, :, 0] = value
        if low:
            lo[at, :, 0] = value
        table = table.clone()
        table[0, missing] = -1
        return Q, lo, hi, table
    return change


# (bounds of a page whose keys hold so low a value in a channel; an infinite upper bound alone)
KINDS = [(torch.bfloat16, -2e38, True), (torch.bfloat16, -1e38, True), (torch.bfloat16, -math.inf, False),
         (torch.float16, -math.inf, False)]



def _check(T, pages, Hq, Hk, D, dtype, counts, ends, change, P=16):
    """One sequence, its last page partly filled."""
    n, lens = pages + 3, [P * pages - 3]
    table = torch.randperm(n, generator=torch.Generator().manual_seed(1))[:pages].view(1, -1).to(torch.int32).cuda()
    mid, wide = L.randn(n, Hk, D, seed=1), 1 + L.randn(n, Hk, D, seed=2).abs()
    Q, lo, hi, table = change(L.randn(T, Hq, D, seed=3, dtype=dtype), (mid - wide).to(dtype), (mid + wide).to(dtype), table)
    for count in counts:
        for first, last in ends:
            print(f"[choice] {pages} pages, {count} of them, {first}/{last}, {T} tokens {Hq}/{Hk} D={D} {dtype}", flush=True)
            got = tdq.tdq_select_pages(Q, lo, hi, L.starts([T]), table, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                       P, count, first=first, last=last)
            want = _choice(Q, lo, hi, [T], lens, table, P, count, first, last, True)
            assert torch.equal(got, want), (got != want).nonzero()[:5].tolist()


@pytest.mark.parametrize("dtype,value,low", KINDS)
@pytest.mark.parametrize("Hq,Hk,D", [(1, 1, 32), (8, 2, 128), (5, 1, 256)])
def test_lowest_scores(Hq, Hk, D, dtype, value, low):
    """A line of few pages, one of more than a workgroup scores, and one of more than stay in registers."""
    for pages in (5, 600, 2100):
        for missing in ([2], [0], [1, pages - 1]):
            there = pages - len(missing)
            for places in ([pages - 2], [3, pages - 2]):
                _check(1, pages, Hq, Hk, D, dtype, (there - 1, there), ((0, 0), (1, 1)), _lowest(low, places, missing, value))


@pytest.mark.parametrize("dtype,value,low", KINDS)
def test_all_scores_among_the_lowest(dtype, value, low):
    """Nothing else than such scores, and pages that are not there."""
    for pages, missing in ((6, [3]), (40, [0, 39]), (700, [350])):
        there = pages - len(missing)
        _check(1, pages, 4, 2, 64, dtype, (there - 2, there), ((0, 0), (0, 1), (2, 1)),
               _lowest(low, list(range(pages)), missing, value))


@pytest.mark.parametrize("dtype,value,low", KINDS)
def test_lowest_scores_of_many_tokens(dtype, value, low):
    """Tokens of a sequence together: those whose pages are as many as are wanted, and fewer."""
    for Hq, Hk in ((32, 32), (64, 32)):
        _check(260, 20, Hq, Hk, 16, dtype, (12, 16), ((1, 1),), _lowest(low, [4, 15], [2], value))
