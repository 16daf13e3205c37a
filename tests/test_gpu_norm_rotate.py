"""Norm of query and key heads with the rotation by position, against 64 bits."""
import pytest
import torch

from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu


def _tol(want, x, dtype):
    """Binary32: the mean of D squares, a root, a quotient, two products, the angle's cosine and the turn, about a
    dozen roundings of numbers no larger than the two of a pair; then the result's own rounding."""
    size = want.abs().amax(dim=-1, keepdim=True)
    return 24 * 2.0 ** -24 * size + L.UNIT[dtype] * want.abs() + L.TINY[dtype]


def _check(T, Hq, Hk, D, R, axes, inter, dtype, norm=True, far=0, fused=True):
    qkv = L.randn(T, Hq + 2 * max(Hk, 1), D, seed=T + D, dtype=dtype)
    Q = qkv[:, :Hq] if fused else qkv[:, :Hq].contiguous()
    K = None if Hk == 0 else qkv[:, Hq:Hq + Hk] if fused else qkv[:, Hq:Hq + Hk].contiguous()
    wq, wk = (1 + 0.2 * L.randn(D, seed=s) for s in (1, 2)) if norm else (None, None)
    P = R // 2
    freq = (10000.0 ** (-torch.arange(P, device="cuda").double() / max(P, 1))).float() if P else None
    axis = (torch.arange(P, device="cuda") % axes).to(torch.int32) if axes > 1 else None
    pos = torch.randint(-far if far else 0, far + 4000, (axes, T), generator=L.gen(3), device="cuda").to(torch.int32)
    got = tdq.tdq_norm_rotate(Q, K, pos if P else None, freq, q_weight=wq, k_weight=wk, axis=axis, interleaved=inter)
    for x, w, y in ((Q, wq, got[0]), (K, wk, got[1])):
        if x is None:
            assert y is None
            continue
        want = L.norm_rotate(x, w, 1e-6, pos, freq, axis, inter)
        bad = ((y.double() - want).abs() / _tol(want, x, dtype)).masked_fill(y.double() == want, 0)
        assert float(bad.max()) <= 1.0, float(bad.max())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,R", [(1, 1, 1, 8, 8), (1, 32, 8, 128, 128), (3, 5, 0, 64, 64), (7, 6, 2, 80, 80),
                                         (50, 4, 4, 96, 48), (17, 3, 1, 256, 256), (9, 2, 2, 40, 16), (11, 7, 7, 72, 8),
                                         (13, 2, 1, 248, 0), (5000, 4, 2, 64, 64), (4097, 3, 1, 32, 32)])
def test_norm_rotate(T, Hq, Hk, D, R, inter, dtype):
    print(f"[norm_rotate] T={T} {Hq}/{Hk} D={D} R={R} {inter} {dtype}", flush=True)
    _check(T, Hq, Hk, D, R, 1, inter, dtype)


@pytest.mark.parametrize("axes", [2, 3])
@pytest.mark.parametrize("inter", [False, True])
def test_axes_and_far_positions(axes, inter):
    _check(300, 4, 2, 96, 96, axes, inter, torch.float32, far=2_000_000)
    _check(300, 4, 2, 64, 32, axes, inter, torch.bfloat16, far=30000, fused=False)


@pytest.mark.parametrize("inter", [False, True])
def test_without_norm(inter):
    _check(40, 4, 2, 64, 64, 1, inter, torch.float16, norm=False)
    _check(40, 4, 2, 64, 64, 1, inter, torch.float32, norm=False)


def test_in_place_and_neighbours():
    """In place in a fused projection: values and what lies between the heads stay as they are."""
    T, Hq, Hk, D = 33, 6, 2, 64
    qkv = L.randn(T, Hq + 2 * Hk + 1, D, seed=8, dtype=torch.bfloat16)
    before = qkv.clone()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freq = (10000.0 ** (-torch.arange(D // 2, device="cuda") / 32.0)).float()
    w = 1 + 0.1 * L.randn(D, seed=1)
    want = tdq.tdq_norm_rotate(qkv[:, :Hq], qkv[:, Hq:Hq + Hk], pos, freq, q_weight=w, k_weight=w)
    tdq.tdq_norm_rotate(qkv[:, :Hq], qkv[:, Hq:Hq + Hk], pos, freq, q_weight=w, k_weight=w,
                        out=(qkv[:, :Hq], qkv[:, Hq:Hq + Hk]))
    assert torch.equal(qkv[:, :Hq], want[0]) and torch.equal(qkv[:, Hq:Hq + Hk], want[1])
    assert torch.equal(qkv[:, Hq + Hk:], before[:, Hq + Hk:])


def test_strides_that_are_not_tokens_first():
    """Heads outermost, and rows that start at an odd element."""
    T, H, D = 20, 3, 32
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freq = (100.0 ** (-torch.arange(D // 2, device="cuda") / 16.0)).float()
    heads_first = L.randn(H, T, D, seed=4, dtype=torch.float16)
    a = tdq.tdq_norm_rotate(heads_first.transpose(0, 1), None, pos, freq)[0]
    b = tdq.tdq_norm_rotate(heads_first.transpose(0, 1).contiguous(), None, pos, freq)[0]
    assert torch.equal(a, b)
    odd = torch.randn((T, 1 + H * D + 2), generator=L.gen(6), device="cuda").half()[:, 1:1 + H * D].unflatten(1, (H, D))
    a = tdq.tdq_norm_rotate(odd, None, pos, freq)[0]
    assert torch.equal(a, tdq.tdq_norm_rotate(odd.contiguous(), None, pos, freq)[0])


def test_zero_and_nan_heads():
    """A head of zeros stays zero; a NaN stays in its own head."""
    T, H, D = 4, 3, 64
    x = L.randn(T, H, D, seed=1, dtype=torch.float16)
    x[1, 1] = 0
    x[2, 0, 5] = float("nan")
    w = torch.ones(D, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    y = tdq.tdq_norm_rotate(x, None, pos, torch.ones(D // 2, device="cuda"), q_weight=w)[0]
    assert bool((y[1, 1] == 0).all())
    assert bool(torch.isnan(y[2, 0]).all())
    ok = torch.ones((T, H), dtype=torch.bool, device="cuda")
    ok[2, 0] = False
    assert torch.isfinite(y[ok]).all()


def test_axis_numbers_outside_the_axes_take_the_nearest():
    T, D = 6, 32
    x = L.randn(T, 2, D, seed=1)
    pos = torch.stack([torch.arange(T), 3 * torch.arange(T)]).to(torch.int32).cuda()
    freq = torch.full((D // 2,), 0.3, device="cuda")
    wild = torch.tensor([-5, 0, 1, 9] * 4, dtype=torch.int32, device="cuda")
    near = torch.tensor([0, 0, 1, 1] * 4, dtype=torch.int32, device="cuda")
    a, b = (tdq.tdq_norm_rotate(x, None, pos, freq, axis=k)[0] for k in (wild, near))
    assert torch.equal(a, b)
