"""Refusals of the operators on a cache in pages: checked on the host, before anything is launched."""
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


def _h(data=FAKE, token=256, head=64):
    return C.byref(tdq.Heads(data, token, head))


def _p(data=FAKE, page=4096, token=256, head=64):
    return C.byref(tdq.Pages(data, page, token, head))


def _s(cu=FAKE, lens=FAKE, table=FAKE, ld=10, S=2, columns=10, n_pages=30, page_size=16):
    return C.byref(tdq.Sequences(cu, lens, table, ld, S, columns, n_pages, page_size))


BAD_SEQUENCES = [(dict(lens=None), tdq.ERR_NULL), (dict(table=None), tdq.ERR_NULL), (dict(S=0), tdq.ERR_SHAPE),
                 (dict(S=(1 << 20) + 1), tdq.ERR_SHAPE), (dict(columns=0), tdq.ERR_SHAPE), (dict(ld=9), tdq.ERR_SHAPE),
                 (dict(n_pages=0), tdq.ERR_SHAPE), (dict(page_size=0), tdq.ERR_SHAPE), (dict(page_size=8), tdq.ERR_SHAPE),
                 (dict(page_size=48), tdq.ERR_SHAPE), (dict(page_size=2048), tdq.ERR_SHAPE),
                 (dict(page_size=-(1 << 31)), tdq.ERR_SHAPE),
                 (dict(columns=(1 << 26) + 1, ld=1 << 27), tdq.ERR_SHAPE), (dict(cu=FAKE + 2), tdq.ERR_ALIGN),
                 (dict(lens=FAKE + 1), tdq.ERR_ALIGN), (dict(table=FAKE + 2), tdq.ERR_ALIGN)]


def _sequences_refused(call, name="seq"):
    assert call(**{name: None}) == tdq.ERR_NULL
    for kw, want in BAD_SEQUENCES:
        assert call(**{name: _s(**kw)}) == want, kw


def test_append():
    ok = dict(Q=_h(), K=_h(), V=_h(), dt=0, T=10, seq=_s(), Hq=4, Hk=2, D=64, wq=None, wk=None, eps=1e-6, R=64, inter=0,
              pos=FAKE, ld_pos=10, axes=1, axis=None, freq=FAKE, Qo=_h(), Kc=_p(), Vc=_p(), st=None)
    call = _caller(tdq.lib().tdq_cache_append, ok)
    for k in ("Q", "K", "V", "Qo"):
        assert call(**{k: None}) == tdq.ERR_NULL and call(**{k: _h(None)}) == tdq.ERR_NULL
    for k in ("Kc", "Vc"):
        assert call(**{k: None}) == tdq.ERR_NULL and call(**{k: _p(None)}) == tdq.ERR_NULL
    assert call(freq=None) == tdq.ERR_NULL and call(seq=_s(cu=None)) == tdq.ERR_NULL
    _sequences_refused(call)
    for dt in (tdq.TDQ_F32, 3, -1):
        assert call(dt=dt) == tdq.ERR_DTYPE
    for kw in (dict(T=0), dict(T=(1 << 30) + 1, ld_pos=1 << 31), dict(Hq=-1), dict(Hk=0), dict(Hq=4090, Hk=4), dict(Hk=2049),
               dict(D=0), dict(D=60), dict(D=264), dict(R=-8), dict(R=72), dict(R=12), dict(axes=0), dict(ld_pos=9)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == tdq.ERR_PARAM
    for kw in (dict(Q=_h(FAKE + 1)), dict(K=_h(FAKE + 1)), dict(V=_h(FAKE + 1)), dict(Qo=_h(FAKE + 1)), dict(Kc=_p(FAKE + 1)),
               dict(Vc=_p(FAKE + 1)), dict(wq=FAKE + 2), dict(wk=FAKE + 2), dict(pos=FAKE + 2), dict(axis=FAKE + 2),
               dict(freq=FAKE + 1)):
        assert call(**kw) == tdq.ERR_ALIGN, kw


def test_bounds():
    call = _caller(tdq.lib().tdq_page_bounds, dict(K=_p(), dt=2, T=10, seq=_s(), Hk=2, D=64, lo=_h(), hi=_h(), st=None))
    assert call(K=None) == tdq.ERR_NULL and call(K=_p(None)) == tdq.ERR_NULL
    for k in ("lo", "hi"):
        assert call(**{k: None}) == tdq.ERR_NULL and call(**{k: _h(None)}) == tdq.ERR_NULL
    _sequences_refused(call)
    assert call(dt=tdq.TDQ_F32) == tdq.ERR_DTYPE
    for kw in (dict(T=-1), dict(T=(1 << 30) + 1), dict(Hk=0), dict(Hk=4097), dict(D=0), dict(D=12), dict(D=264)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    for kw in (dict(K=_p(FAKE + 1)), dict(lo=_h(FAKE + 1)), dict(hi=_h(FAKE + 1))):
        assert call(**kw) == tdq.ERR_ALIGN, kw


ATTENTION_SHAPES = [dict(Tq=0), dict(Tq=(1 << 30) + 1), dict(Hq=0), dict(Hk=0), dict(Hq=5), dict(Hq=8192), dict(D=0),
                    dict(D=20), dict(D=264)]


def test_select():
    L = tdq.lib()
    call = _caller(L.tdq_select_pages, dict(Q=_h(), lo=_h(), hi=_h(), dt=0, Tq=10, seq=_s(), Hq=4, Hk=2, D=64, causal=1, first=1,
                                            last=1, count=4, out=FAKE, ws=FAKE, wsb=1 << 40, st=None))
    for k in ("Q", "lo", "hi"):
        assert call(**{k: None}) == tdq.ERR_NULL and call(**{k: _h(None)}) == tdq.ERR_NULL
    assert call(out=None) == tdq.ERR_NULL and call(seq=_s(cu=None)) == tdq.ERR_NULL
    _sequences_refused(call)
    assert call(dt=tdq.TDQ_F32) == tdq.ERR_DTYPE
    for kw in ATTENTION_SHAPES:
        assert call(**kw) == tdq.ERR_SHAPE, kw
    for kw in (dict(count=0, first=0, last=0), dict(count=(1 << 20) + 1), dict(first=-1), dict(last=-1), dict(count=1),
               dict(first=(1 << 31) - 1, last=(1 << 31) - 1)):
        assert call(**kw) == tdq.ERR_PARAM, kw
    for kw in (dict(Q=_h(FAKE + 1)), dict(lo=_h(FAKE + 1)), dict(hi=_h(FAKE + 1)), dict(out=FAKE + 2)):
        assert call(**kw) == tdq.ERR_ALIGN, kw
    assert call(Tq=1 << 30, Hq=4096, Hk=4096, seq=_s(columns=1 << 20, ld=1 << 20)) == tdq.ERR_SHAPE
    need = L.tdq_select_pages_workspace_bytes(10, 2, 10)
    assert need >= 10 * 2 * 10 * 4
    for kw in (dict(ws=None), dict(wsb=need - 1), dict(ws=FAKE + 128)):
        assert call(**kw) == tdq.ERR_WORKSPACE, kw
    for a in ((0, 2, 10), (1 << 31, 2, 10), (10, 0, 10), (10, 5000, 10), (10, 2, 0), (10, 2, 1 << 27), (1 << 30, 4096, 1 << 20)):
        assert L.tdq_select_pages_workspace_bytes(*a) == 0


def test_selected():
    L = tdq.lib()
    call = _caller(L.tdq_attention_selected, dict(Q=_h(), K=_p(), V=_p(), dt=0, Tq=10, seq=_s(), Hq=4, Hk=2, D=64, scale=0.125,
                                                  causal=1, chosen=FAKE, count=64, O=_h(), lse=None, ws=FAKE, wsb=1 << 40, st=None))
    _attention(call)
    assert call(chosen=None) == tdq.ERR_NULL and call(chosen=FAKE + 2) == tdq.ERR_ALIGN
    for kw in (dict(count=0), dict(count=(1 << 20) + 1), dict(count=1 << 20, seq=_s(page_size=1024, n_pages=5), Tq=0)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    need = L.tdq_attention_selected_workspace_bytes(10, 4, 2, 64, 16, 64)
    assert need > 0
    for kw in (dict(ws=None), dict(wsb=need - 1), dict(ws=FAKE + 128)):
        assert call(**kw) == tdq.ERR_WORKSPACE, kw
    assert L.tdq_attention_selected_workspace_bytes(10, 4, 2, 64, 16, 1) == 0
    for a in ((0, 4, 2, 64, 16, 64), (10, 5, 2, 64, 16, 64), (10, 4, 2, 60, 16, 64), (10, 4, 2, 64, 24, 64), (10, 4, 2, 64, 16, 0)):
        assert L.tdq_attention_selected_workspace_bytes(*a) == 0


def _attention(call):
    for k, bad in (("Q", _h), ("O", _h), ("K", _p), ("V", _p)):
        assert call(**{k: None}) == tdq.ERR_NULL and call(**{k: bad(None)}) == tdq.ERR_NULL
        for kw in (dict(data=FAKE + 8), dict(token=260), dict(head=60)) + ((dict(page=4100),) if bad is _p else ()):
            assert call(**{k: bad(**kw)}) == tdq.ERR_ALIGN, (k, kw)
    assert call(lse=FAKE + 2) == tdq.ERR_ALIGN and call(seq=_s(cu=None)) == tdq.ERR_NULL
    _sequences_refused(call)
    for dt in (tdq.TDQ_F32, 3):
        assert call(dt=dt) == tdq.ERR_DTYPE
    for kw in ATTENTION_SHAPES:
        assert call(**kw) == tdq.ERR_SHAPE, kw
    for scale in (float("nan"), float("inf")):
        assert call(scale=scale) == tdq.ERR_PARAM


def test_paged():
    L = tdq.lib()
    call = _caller(L.tdq_attention_paged, dict(Q=_h(), K=_p(), V=_p(), dt=0, Tq=10, seq=_s(), prefix=_s(S=1), Hq=4, Hk=2, D=64,
                                               scale=0.125, causal=1, O=_h(), lse=None, ws=FAKE, wsb=1 << 50, st=None))
    _attention(call)
    for kw, want in BAD_SEQUENCES:
        assert call(prefix=_s(**kw)) == want, kw
    assert call(prefix=_s(cu=None)) == tdq.ERR_NULL
    for kw in (dict(prefix=_s(page_size=32)), dict(prefix=_s(n_pages=31)), dict(Tq=1 << 30, Hq=8, Hk=2)):
        assert call(**kw) == tdq.ERR_SHAPE, kw
    need = L.tdq_attention_paged_workspace_bytes(10, 2, 1, 4, 2, 64)
    assert need > L.tdq_attention_paged_workspace_bytes(10, 2, 0, 4, 2, 64) > 0
    for kw in (dict(ws=None), dict(wsb=need - 1), dict(ws=FAKE + 128)):
        assert call(**kw) == tdq.ERR_WORKSPACE, kw
    for a in ((0, 2, 1, 4, 2, 64), (10, 0, 1, 4, 2, 64), (10, 2, -1, 4, 2, 64), (10, 2, 1, 5, 2, 64), (10, 2, 1, 4, 2, 60),
              (1 << 30, 2, 0, 8, 2, 64), (10, (1 << 20) + 1, 0, 4, 2, 64)):
        assert L.tdq_attention_paged_workspace_bytes(*a) == 0


def test_binding_refuses_what_does_not_fit():
    t = lambda *s, dt=torch.float16: torch.zeros(s, dtype=dt)
    i = lambda *s: t(*s, dt=torch.int32)
    x, kv, c, f = t(5, 4, 16), t(5, 2, 16), t(3, 16, 2, 16), t(8, dt=torch.float32)
    seq = (i(3), i(2, 4), i(2))
    append = lambda **kw: tdq.tdq_cache_append(**dict(dict(Q=x, K=kv, V=kv, cache_k=c, cache_v=c, cu_q=seq[0], table=seq[1],
                                                           len_k=seq[2], freq=f), **kw))
    for kw in (dict(Q=t(4, 4, 16)), dict(Q=t(5, 4, 8)), dict(V=t(5, 2, 8)), dict(V=t(4, 2, 16)), dict(cache_k=t(3, 16, 16)),
               dict(cache_k=t(3, 16, 4, 16)), dict(cache_v=t(4, 16, 2, 16)), dict(cache_k=c.bfloat16()), dict(cu_q=i(4)),
               dict(len_k=i(3)), dict(table=i(8)), dict(table=i(4, 2).t()), dict(pos=i(4)), dict(q_weight=t(15, dt=torch.float32)),
               dict(k_weight=t(16)), dict(axis=i(7)), dict(out=t(5, 4, 8)), dict(out=x.bfloat16()),
               dict()):                                              # (on the host)
        with pytest.raises(ValueError):
            append(**kw)
    for kw in (dict(cu_q=seq[0].long()), dict(len_k=seq[2].long()), dict(table=seq[1].long()), dict(freq=f.half()),
               dict(pos=i(5).long()), dict(axis=i(8).long())):
        with pytest.raises(TypeError):
            append(**kw)
    for kw in (dict(cu_q=seq[0]), dict(out=(t(3, 2, 16), t(3, 2, 8))), dict(out=(t(3, 2, 16), t(3, 2, 16).bfloat16())), dict()):
        with pytest.raises(ValueError):
            tdq.tdq_page_bounds(c, seq[1], seq[2], **kw)
    b = t(3, 2, 16)
    select = lambda **kw: tdq.tdq_select_pages(**dict(dict(Q=x, lo=b, hi=b, cu_q=seq[0], table=seq[1], len_k=seq[2], page_size=16,
                                                           count=4), **kw))
    for kw in (dict(lo=t(3, 2, 8)), dict(hi=t(4, 2, 16)), dict(hi=b.bfloat16()), dict(out=i(5, 2, 3)), dict(out=t(5, 2, 4)),
               dict(workspace=t(64, 2, dt=torch.uint8).t()), dict()):
        with pytest.raises(ValueError):
            select(**kw)
    base = dict(Q=x, cache_k=c, cache_v=c, cu_q=seq[0], table=seq[1], len_k=seq[2])
    bad = [dict(cache_k=t(3, 16, 2, 8)), dict(cache_v=t(3, 16, 2, 16).bfloat16()), dict(cache_v=t(3, 32, 2, 16)),
           dict(out=t(5, 4, 8)), dict(lse=t(5, 3, dt=torch.float32)), dict(lse=t(5, 4)), dict(len_k=i(3)), dict()]
    for kw in bad + [dict(prefix=(i(2), i(1, 2))), dict(prefix=(i(3), i(1, 2), i(1))), dict(prefix=(i(2), i(1, 2), i(2)))]:
        with pytest.raises(ValueError):
            tdq.tdq_attention_paged(**dict(base, **kw))
    with pytest.raises(TypeError):
        tdq.tdq_attention_paged(**base, prefix=(i(2).long(), i(1, 2), i(1)))
    for kw in bad + [dict(chosen=i(4, 2, 3)), dict(chosen=i(5, 4, 3)), dict(chosen=i(5, 2)), dict(chosen=i(5, 3, 2).transpose(1, 2))]:
        with pytest.raises(ValueError):
            tdq.tdq_attention_selected(**dict(dict(base, chosen=i(5, 2, 3)), **kw))
    with pytest.raises(TypeError):
        tdq.tdq_attention_selected(**base, chosen=i(5, 2, 3).long())
