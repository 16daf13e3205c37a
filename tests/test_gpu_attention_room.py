"""Attention over a cache that leaves every sequence room to grow."""
import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq", [1, 3, 40])
def test_lengths_beyond_the_room_are_all_of_it(nq):
    """len_k past a sequence's room means the room, with finite keys: the same as without len_k, bit for bit."""
    S, room, Hq, Hk, D = 4, 300, 4, 2, 64
    Q = L.randn(S * nq, Hq, D, seed=1, dtype=torch.bfloat16)
    K, V = (L.randn(S * room, Hk, D, seed=s, dtype=torch.bfloat16) for s in (2, 3))
    cu_q, cu_k = L.starts([nq] * S), L.starts([room] * S)
    want = tdq.tdq_attention(Q, K, V, cu_q, cu_k, want_lse=True)
    for n in ([room] * S, [room + 1] * S, [room, 10 * room, 2 ** 31 - 1, room + 64]):
        got = tdq.tdq_attention(Q, K, V, cu_q, cu_k, len_k=torch.tensor(n, dtype=torch.int32, device="cuda"), want_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    n = [room + 5, 0, 7, -3]
    got = tdq.tdq_attention(Q, K, V, cu_q, cu_k, len_k=torch.tensor(n, dtype=torch.int32, device="cuda"), want_lse=True)
    used = [min(max(x, 0), room) for x in n]
    keep = torch.cat([torch.arange(s * room, s * room + x, device="cuda") for s, x in enumerate(used)])
    L.check_attention(got, L.attention(Q, K[keep], V[keep], [nq] * S, used, D ** -0.5, True))
