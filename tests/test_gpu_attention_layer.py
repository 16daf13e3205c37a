"""The operators together: an attention layer against the same steps in 64 bits, whole prompts and token by token."""
import pytest
import torch

from paper_2604_16855_amd import attention_layer as A
from paper_2604_16855_amd import tdq

import layer_util as L

pytestmark = pytest.mark.gpu


def _quantized(x, rows):
    """What the codes of x stand for, in 64 bits."""
    codes, step = L.block_codes(x.float(), rows)
    R, K = x.shape
    return L.code_values(codes, K) * step.double().repeat_interleave(rows, 0).repeat_interleave(128, 1)[:R, :K]


def _layer(C, Hq, Hk, D, axes):
    freq = (10000.0 ** (-torch.arange(D // 2, device="cuda").double() / (D // 2))).float()
    axis = (torch.arange(D // 2, device="cuda") % axes).to(torch.int32) if axes > 1 else None
    w1, w2 = 0.02 * L.randn((Hq + 2 * Hk) * D, C, seed=1), 0.02 * L.randn(C, Hq * D, seed=2)
    qn, kn = 1 + 0.1 * L.randn(D, seed=3), 1 + 0.1 * L.randn(D, seed=4)
    return A.AttentionLayer(w1, w2, Hq, Hk, D, freq, axis=axis, q_norm=qn, k_norm=kn, causal=axes == 1), w1, w2


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("C,Hq,Hk,D,axes,lengths", [(200, 4, 2, 64, 1, [70, 1, 133]), (512, 8, 8, 32, 2, [49, 196, 121])])
def test_layer(C, Hq, Hk, D, axes, lengths, dtype):
    layer, w1, w2 = _layer(C, Hq, Hk, D, axes)
    T = sum(lengths)
    X = L.randn(T, C, seed=5, dtype=dtype)
    pos = torch.randint(0, 200, (axes, T), generator=L.gen(6), device="cuda").to(torch.int32)
    got = layer(X, pos, L.starts(lengths)).double()
    y = (_quantized(X, 1) @ _quantized(w1, 128).t().contiguous()).unflatten(1, (-1, D))
    rot = lambda x, w: L.norm_rotate(x, w, 1e-6, pos, layer.freq, layer.axis, False)
    Q, K, V = rot(y[:, :Hq], layer.q_norm), rot(y[:, Hq:Hq + Hk], layer.k_norm), y[:, Hq + Hk:]
    O = L.attention(Q.to(dtype), K.to(dtype), V.to(dtype), lengths, lengths, D ** -0.5, axes == 1)[0].flatten(1)
    want = _quantized(O, 1) @ _quantized(w2, 128).t().contiguous()
    # The layer rounds four times to the type (projection, heads, probabilities, output of the attention), half a unit
    # each, and a rounding that changes sides in front of the second quantizer moves a code of 3 fraction bits, 2^-4 at
    # most: of values that differ by d some d / 2^-4 change sides, which in the norm is sqrt(d 2^-4).
    d = 4 * L.UNIT[dtype]
    tol = d + (d * 2.0 ** -4) ** 0.5
    err = float((got - want).norm() / want.norm())
    print(f"[layer] {lengths} {dtype} error {err:.1e} of {tol:.1e}", flush=True)
    assert err <= tol


def test_token_by_token():
    layer, _, _ = _layer(256, 4, 2, 64, 1)
    lengths, more = [40, 3, 129], 3
    X = [L.randn(n + more, 256, seed=i, dtype=torch.bfloat16) for i, n in enumerate(lengths)]

    def run(counts, first, step):
        x = torch.cat([v[f:f + n] for v, n, f in zip(X, counts, first)])
        pos = torch.cat([torch.arange(f, f + n, device="cuda") for n, f in zip(counts, first)]).to(torch.int32)
        return step(x, pos, L.starts(counts))

    whole = run([n + more for n in lengths], [0] * 3, layer)
    cache = A.Cache(3, 200, 2, 64, torch.bfloat16, "cuda")
    parts = [run(lengths, [0] * 3, lambda *a: layer.step(*a, cache))]
    for i in range(more):
        parts.append(run([1] * 3, [n + i for n in lengths], lambda *a: layer.step(*a, cache)))
    assert cache.used.tolist() == [n + more for n in lengths]
    ends = L.starts([n + more for n in lengths])[1:].tolist()
    # the same sums in another order: rounded differently now and then, which moves a code in front of the projection
    d = 2 * L.UNIT[torch.bfloat16]
    tol = d + (d * 2.0 ** -4) ** 0.5
    for i in range(more):
        want = torch.stack([whole[e - more + i] for e in ends]).double()
        err = float((parts[1 + i].double() - want).norm() / want.norm())
        assert err <= tol, err


def test_example_runs(capsys):
    A.main()
    assert "relative difference" in capsys.readouterr().out


def test_layer_under_a_graph():
    """The layer captured once and replayed on new inputs gives what it gives directly."""
    layer, _, _ = _layer(256, 4, 2, 64, 1)
    lengths = [1] * 6
    cu_k = L.starts([700, 1, 64, 2000, 333, 5])
    K, V = L.randn(3103, 2, 64, seed=1, dtype=torch.bfloat16), L.randn(3103, 2, 64, seed=2, dtype=torch.bfloat16)
    X, cu = L.randn(6, 256, seed=3, dtype=torch.bfloat16), L.starts(lengths)
    pos = torch.arange(6, dtype=torch.int32, device="cuda")

    def call():
        Q, _, _ = layer._heads(X, pos)
        return layer._project(tdq.tdq_attention(Q, K, V, cu, cu_k)[0])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
    for seed in range(3):
        X.copy_(L.randn(6, 256, seed=10 + seed, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, call())
        torch.cuda.synchronize()
