"""Refusals of the 8-bit linear, the head norm and the attention: checked on the host, before anything is launched."""
import ctypes as C
import os

import pytest
import torch

from paper_2604_16855_amd import tdq

pytestmark = pytest.mark.skipif(not os.path.exists(tdq.LIB_PATH),
                                reason="libtdq.so not built (python -m paper_2604_16855_amd.build)")

FAKE = 4096   # a non-null, aligned "device pointer"; never dereferenced by a failing call


def _caller(f, ok):
    def call(**kw):
        a = dict(ok, **kw)
        assert set(a) == set(ok)
        return f(*a.values())
    return call


@pytest.mark.parametrize("name", ["tdq_quantize_act_f8", "tdq_quantize_weight_f8"])
def test_quantizers(name):
    call = _caller(getattr(tdq.lib(), name), dict(X=FAKE, dt=0, M=8, K=200, ld=200, Q=FAKE, ld_q=208, s=FAKE, ld_s=2,
                                                  st=None))
    for k in ("X", "Q", "s"):
        assert call(**{k: None}) == tdq.ERR_NULL
    assert call(dt=3) == tdq.ERR_DTYPE
    for kw in (dict(M=0), dict(M=(1 << 30) + 1), dict(K=0), dict(K=131073, ld=131073, ld_q=131088, ld_s=1025),
               dict(ld=199), dict(ld_q=192), dict(ld_s=1)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    assert call(M=1 << 26, K=4096, ld=4096, ld_q=4096, ld_s=32) == tdq.ERR_SHAPE      # 2^31 blocks
    for kw in (dict(X=FAKE + 1), dict(Q=FAKE + 8), dict(ld_q=216), dict(s=FAKE + 2)):
        assert call(**kw) == tdq.ERR_ALIGN, kw
    assert call(dt=tdq.TDQ_F32, X=FAKE + 2) == tdq.ERR_ALIGN
    if "weight" in name:
        assert call(M=(1 << 22) + 1) == tdq.ERR_SHAPE


def test_linear():
    call = _caller(tdq.lib().tdq_linear_f8,
                   dict(Qx=FAKE, ld_q=208, xs=FAKE, ld_xs=2, M=8, K=200, N=130, Qw=FAKE, ld_w=208, ws=FAKE, ld_ws=2,
                        b=None, Y=FAKE, dt=0, ld_y=130, st=None))
    for k in ("Qx", "xs", "Qw", "ws", "Y"):
        assert call(**{k: None}) == tdq.ERR_NULL
    assert call(dt=3) == tdq.ERR_DTYPE
    for kw in (dict(M=0), dict(M=(1 << 30) + 1), dict(K=0), dict(N=0), dict(N=(1 << 22) + 1, ld_y=1 << 23),
               dict(ld_q=192), dict(ld_w=192), dict(ld_xs=1), dict(ld_ws=1), dict(ld_y=129),
               dict(ld_q=(1 << 22) + 16), dict(ld_w=(1 << 22) + 16), dict(ld_xs=(1 << 20) + 1)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    for kw in (dict(Qx=FAKE + 8), dict(Qw=FAKE + 4), dict(ld_q=200), dict(ld_w=216), dict(xs=FAKE + 2),
               dict(ws=FAKE + 1), dict(b=FAKE + 2), dict(Y=FAKE + 1), dict(dt=tdq.TDQ_F32, Y=FAKE + 2)):
        assert call(**kw) == tdq.ERR_ALIGN, kw


def _h(data=FAKE, token=256, head=64):
    return C.byref(tdq.Heads(data, token, head))


def test_norm_rotate():
    ok = dict(Q=_h(), K=_h(), dt=2, T=10, Hq=4, Hk=2, D=64, wq=FAKE, wk=FAKE, eps=1e-6, R=64, inter=0, pos=FAKE,
              ld_pos=10, axes=1, axis=None, freq=FAKE, Qo=_h(), Ko=_h(), st=None)
    call = _caller(tdq.lib().tdq_norm_rotate, ok)
    for kw in (dict(Q=None), dict(Qo=None), dict(Q=_h(None)), dict(Qo=_h(None)), dict(K=None), dict(Ko=None),
               dict(K=_h(None)), dict(pos=None), dict(freq=None)):
        assert call(**kw) == tdq.ERR_NULL, kw
    assert call(dt=7) == tdq.ERR_DTYPE
    for kw in (dict(T=0), dict(T=(1 << 30) + 1, ld_pos=1 << 31), dict(Hq=0), dict(Hk=-1), dict(Hq=4095), dict(D=0),
               dict(D=60), dict(D=264), dict(R=-8), dict(R=72), dict(R=12), dict(axes=0), dict(ld_pos=9)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == tdq.ERR_PARAM
    for kw in (dict(Q=_h(FAKE + 1)), dict(K=_h(FAKE + 1)), dict(Qo=_h(FAKE + 1)), dict(Ko=_h(FAKE + 1)),
               dict(wq=FAKE + 2), dict(wk=FAKE + 2), dict(pos=FAKE + 2), dict(axis=FAKE + 2), dict(freq=FAKE + 1),
               dict(dt=tdq.TDQ_F32, Q=_h(FAKE + 2))):
        assert call(**kw) == tdq.ERR_ALIGN, kw


def test_attention():
    L = tdq.lib()
    ok = dict(Q=_h(), K=_h(), V=_h(), dt=0, Tq=10, Tk=20, S=2, cq=FAKE, ck=FAKE, lk=None, Hq=4, Hk=2, D=64, scale=0.125,
              causal=1, O=_h(), lse=None, ws=FAKE, wsb=1 << 40, st=None)
    call = _caller(L.tdq_attention, ok)
    for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(cq=None), dict(ck=None), dict(Q=_h(None)),
               dict(K=_h(None)), dict(V=_h(None)), dict(O=_h(None))):
        assert call(**kw) == tdq.ERR_NULL, kw
    for dt in (tdq.TDQ_F32, 3):
        assert call(dt=dt) == tdq.ERR_DTYPE
    shapes = (dict(Tq=0), dict(Tq=(1 << 30) + 1), dict(Tk=-1), dict(Tk=(1 << 30) + 1), dict(S=0), dict(S=(1 << 20) + 1),
              dict(Hq=0), dict(Hk=0), dict(Hq=5), dict(Hq=8192), dict(D=0), dict(D=20), dict(D=264))
    for kw in shapes:
        assert call(**kw) == tdq.ERR_SHAPE, kw
        a = dict(Tq=10, Tk=20, S=2, Hq=4, Hk=2, D=64)
        a.update(kw)
        assert L.tdq_attention_workspace_bytes(*a.values()) == 0
    for scale in (float("nan"), float("inf")):
        assert call(scale=scale) == tdq.ERR_PARAM
    for k in ("Q", "K", "V", "O"):
        for bad in (_h(FAKE + 8), _h(token=260), _h(head=60)):
            assert call(**{k: bad}) == tdq.ERR_ALIGN
    for kw in (dict(cq=FAKE + 2), dict(ck=FAKE + 2), dict(lk=FAKE + 2), dict(lse=FAKE + 2)):
        assert call(**kw) == tdq.ERR_ALIGN, kw


def test_attention_workspace():
    """Where the call needs scratch, none, too little or a misaligned one is refused."""
    L = tdq.lib()
    shape = (1, 100000, 1, 8, 8, 128)
    need = L.tdq_attention_workspace_bytes(*shape)
    if need:
        for ws, n in ((None, need), (FAKE, need - 1), (FAKE + 128, need)):
            assert L.tdq_attention(_h(), _h(), _h(), 0, 1, 100000, 1, FAKE, FAKE, None, 8, 8, 128, 0.1, 1, _h(), None, ws, n,
                                   None) == tdq.ERR_WORKSPACE


def test_binding_refuses_what_does_not_fit():
    t = lambda *s, dt=torch.float16: torch.zeros(s, dtype=dt)
    with pytest.raises(TypeError):
        tdq.tdq_quantize_act_f8(t(4, 8, dt=torch.int32))
    with pytest.raises(ValueError):
        tdq.tdq_quantize_act_f8(t(8, 4).t())
    with pytest.raises(ValueError):
        tdq.tdq_quantize_act_f8(t(4, 20), out=(t(4, 16, dt=torch.uint8), t(4, 1, dt=torch.float32)))
    q, s = t(4, 32, dt=torch.uint8), t(4, 1, dt=torch.float32)
    with pytest.raises(TypeError):
        tdq.tdq_linear_f8(q.to(torch.int8), s, 32, q, s)
    with pytest.raises(ValueError):
        tdq.tdq_linear_f8(q, s, 32, q, s, bias=t(5, dt=torch.float32))
    with pytest.raises(ValueError):
        tdq.tdq_linear_f8(q, s, 32, q, s, out=t(4, 3))
    with pytest.raises(ValueError):
        tdq.tdq_linear_f8(q, s[:3], 32, q, s)
    x, p, f = t(5, 2, 16), t(5, dt=torch.int32), t(8, dt=torch.float32)
    with pytest.raises(ValueError):
        tdq.tdq_norm_rotate(x, t(4, 2, 16), p, f)
    with pytest.raises(TypeError):
        tdq.tdq_norm_rotate(x, x, p.long(), f)
    with pytest.raises(ValueError):
        tdq.tdq_norm_rotate(x, x, p[:4], f)
    with pytest.raises(ValueError):
        tdq.tdq_norm_rotate(x, x, p, f, q_weight=t(15, dt=torch.float32))
    with pytest.raises(ValueError):
        tdq.tdq_norm_rotate(x, x, p, f, axis=t(7, dt=torch.int32))
    c = t(2, dt=torch.int32)
    with pytest.raises(ValueError):
        tdq.tdq_attention(x, x, t(4, 2, 16), c, c)
    with pytest.raises(ValueError):
        tdq.tdq_attention(x, x, x, c, t(3, dt=torch.int32))
    with pytest.raises(TypeError):
        tdq.tdq_attention(x, x, x, c.long(), c)
    with pytest.raises(ValueError):
        tdq.tdq_attention(x, x, x, c, c, lse=t(5, 3, dt=torch.float32))
    with pytest.raises(ValueError):
        tdq.tdq_attention(x, x, x, c, c, len_k=t(2, dt=torch.int32))
    with pytest.raises(TypeError):
        tdq.tdq_attention(x, x, x, c, c, len_k=t(1, dt=torch.int64))
