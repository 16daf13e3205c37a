"""The sums of the 8-bit linear."""
import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,N", [(1, 200, 40), (7, 8190, 48), (16, 1024, 130), (32, 4097, 33), (33, 8190, 200),
                                   (512, 512, 300), (1300, 1300, 1000), (8192, 300, 8192)])
def test_every_channel_counts(M, K, N, dtype):
    """Token m has one channel that is not zero, so that Y[m] is one column of the weight: exact but for the step's and
    the result's rounding."""
    g = L.gen(M + K)
    at = (torch.arange(M, device="cuda") * max(1, K // M) + (K - 1 if M == 1 else 0)) % K
    X = torch.zeros((M, K), device="cuda")
    X[torch.arange(M, device="cuda"), at] = 448.0            # (step 1, code 448)
    qx, xs = tdq.tdq_quantize_act_f8(X)
    qw, ws = tdq.tdq_quantize_weight_f8(torch.randn((N, K), generator=g, device="cuda"))
    y = tdq.tdq_linear_f8(qx, xs, K, qw, ws, out_dtype=dtype)
    out = torch.arange(N, device="cuda") // 128
    step = xs.double()[torch.arange(M, device="cuda"), at // 128][:, None] * ws.double()[:, at // 128].t()[:, out]
    want = 448.0 * L.code_values(qw, K).t().contiguous()[at] * step
    tol = (L.UNIT[dtype] + 3 * 2.0 ** -24) * want.abs() + L.TINY[dtype]
    assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("K,N", [(1025, 64), (4096, 200), (8190, 640)])
def test_few_and_more_tokens_agree(K, N, dtype):
    """Up to 32 tokens the blocks of K are added in eight partial sums: the same within the bound of either order."""
    X = L.randn(33, K, seed=K)
    qx, xs = tdq.tdq_quantize_act_f8(X)
    qw, ws = tdq.tdq_quantize_weight_f8(0.05 * L.randn(N, K, seed=2))
    more = tdq.tdq_linear_f8(qx, xs, K, qw, ws, out_dtype=dtype).double()
    _, mag = L.linear(qx, xs, K, qw, ws)
    tol = 2 * (-(-K // 128) + 128 + 4) * 2.0 ** -24 * mag
    if dtype != torch.float32:
        tol = tol + 2 * 2.0 ** -13 * mag + 2 * L.UNIT[dtype] * more.abs() + L.TINY[dtype]
    for M in (32, 16, 1):
        few = tdq.tdq_linear_f8(qx[:M], xs[:M], K, qw, ws, out_dtype=dtype).double()
        assert bool(((few - more[:M]).abs() <= tol[:M]).all())
