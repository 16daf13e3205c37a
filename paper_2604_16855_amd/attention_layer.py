"""An attention layer on the library's operators: projections in 8-bit floating point, the norm and rotation of its
heads, attention over packed sequences, and single tokens over a cache.

    python -m paper_2604_16855_amd.attention_layer        # a prompt, then tokens one at a time

The layer holds the codes and steps of its two weights and nothing else; activations are quantized in front of each
projection.  Everything runs in the library's kernels on the current stream, apart from writing new keys and values to
the cache.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import tdq


class AttentionLayer:
    """Y = attention(rotate(norm(X Wqkv^T))) Wout^T for tokens X[T, C].

    w_qkv [(Hq + 2 Hk) D, C], w_out [C, Hq D]; q_norm, k_norm [D] or None; freq [R / 2] angle per position, axis
    [R / 2] which position axis turns a pair (None: the first)."""

    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, Hq: int, Hk: int, D: int, freq: torch.Tensor,
                 axis: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None,
                 k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                 causal: bool = True):
        if w_qkv.shape[0] != (Hq + 2 * Hk) * D or w_out.shape[1] != Hq * D:
            raise ValueError("the weights do not fit the heads")
        self.qkv, self.out = tdq.tdq_quantize_weight_f8(w_qkv), tdq.tdq_quantize_weight_f8(w_out)
        self.C, self.Hq, self.Hk, self.D = w_qkv.shape[1], Hq, Hk, D
        self.freq, self.axis, self.q_norm, self.k_norm = freq, axis, q_norm, k_norm
        self.eps, self.interleaved, self.causal = eps, interleaved, causal

    def _heads(self, X: torch.Tensor, pos: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """Q[T, Hq, D], K and V[T, Hk, D]: parts of one projection, queries and keys normed and turned in place."""
        codes, step = tdq.tdq_quantize_act_f8(X)
        y = tdq.tdq_linear_f8(codes, step, self.C, *self.qkv, out_dtype=X.dtype).unflatten(1, (-1, self.D))
        Q, K, V = y[:, :self.Hq], y[:, self.Hq:self.Hq + self.Hk], y[:, self.Hq + self.Hk:]
        tdq.tdq_norm_rotate(Q, K, pos, self.freq, q_weight=self.q_norm, k_weight=self.k_norm, eps=self.eps,
                            axis=self.axis, interleaved=self.interleaved, out=(Q, K))
        return Q, K, V

    def _project(self, O: torch.Tensor) -> torch.Tensor:
        codes, step = tdq.tdq_quantize_act_f8(O.flatten(1))
        return tdq.tdq_linear_f8(codes, step, self.Hq * self.D, *self.out, out_dtype=O.dtype)

    def __call__(self, X: torch.Tensor, pos: torch.Tensor, cu: torch.Tensor) -> torch.Tensor:
        """Whole sequences, packed: X[T, C], pos [axes, T] int32, cu [S + 1] int32."""
        Q, K, V = self._heads(X, pos)
        return self._project(tdq.tdq_attention(Q, K, V, cu, cu, causal=self.causal)[0])

    def step(self, X: torch.Tensor, pos: torch.Tensor, cu: torch.Tensor, cache: "Cache") -> torch.Tensor:
        """The next tokens of every sequence of a cache: X[T, C], packed by cu [S + 1]; their keys and values join it
        (refused where a sequence has no room for them)."""
        Q, K, V = self._heads(X, pos)
        cache.append(K, V, cu)
        O, _ = tdq.tdq_attention(Q, cache.K, cache.V, cu, cache.cu, len_k=cache.used, causal=self.causal)
        return self._project(O)


class Cache:
    """Keys and values of S sequences, `room` tokens each, and how many are there."""

    def __init__(self, S: int, room: int, Hk: int, D: int, dtype, device):
        # (a row behind the last sequence takes what has no place)
        self._K = torch.empty((S * room + 1, Hk, D), dtype=dtype, device=device)
        self._V = torch.empty_like(self._K)
        self.K, self.V = self._K[:-1], self._V[:-1]
        self.S, self.room = S, room
        self.cu = room * torch.arange(S + 1, dtype=torch.int32, device=device)
        # one entry more: tokens that belong to no sequence, which fit nowhere
        self._first = self.cu.long()
        self._end = torch.cat([self._first[1:], torch.full_like(self._first[:1], -(1 << 62))])
        self._used = torch.zeros_like(self.cu)
        self.used = self._used[:-1]
        self._most = 0                   # no sequence has more tokens, as far as the host can tell

    def append(self, K: torch.Tensor, V: torch.Tensor, cu: torch.Tensor) -> None:
        """New tokens of every sequence, packed by cu [S + 1] from 0 on.  A sequence without room for its own is
        refused, and the cache left as it is.  The host counts T more for every sequence; only when that would not fit
        does it ask the device for the true numbers.  (A replayed graph does not ask: there, what has no room is left
        out, and the next call that asks is refused.)"""
        T = K.shape[0]
        if cu.shape != (self.S + 1,) or V.shape[0] != T:
            raise ValueError("cu must be one longer than the number of sequences, K and V as long as each other")
        most = self._most + T
        if most > self.room:
            new = cu.tolist()
            total = [u + b - a for u, a, b in zip(self.used.tolist(), new, new[1:])]
            most = max(total)
            if most > self.room:
                raise ValueError(f"sequence {total.index(most)} would have {most} tokens in a room of {self.room}")
        self._write(K, V, cu)
        self._most = most

    def _write(self, K: torch.Tensor, V: torch.Tensor, cu: torch.Tensor) -> None:
        t = torch.arange(K.shape[0], dtype=torch.int32, device=K.device)
        s = torch.searchsorted(cu, t, right=True).sub_(1)        # (in front of the first: -1, the last entry as well)
        at = (self._first + self._used - cu)[s] + t
        at = torch.where(at < self._end[s], at, self.S * self.room)
        self._K.index_copy_(0, at, K)
        self._V.index_copy_(0, at, V)
        self.used += cu[1:] - cu[:-1]


def main() -> None:
    if not torch.cuda.is_available():
        raise SystemExit("the example needs a GPU")
    g = torch.Generator(device="cuda").manual_seed(0)
    C, Hq, Hk, D, lengths, more = 1024, 16, 4, 64, [300, 17, 1024], 8
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    ones = torch.ones(D, device="cuda")
    freq = (10000.0 ** (-torch.arange(D // 2, device="cuda").double() / (D // 2))).float()
    layer = AttentionLayer(0.02 * randn((Hq + 2 * Hk) * D, C), 0.02 * randn(C, Hq * D), Hq, Hk, D, freq, q_norm=ones,
                           k_norm=ones)
    whole = [randn(n + more, C).bfloat16() for n in lengths]
    pack = lambda a, b: torch.cat([x[n + a if a >= 0 else 0:n + b] for x, n in zip(whole, lengths)])  # noqa: E731

    def places(counts, first):
        cu = torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)
        pos = torch.cat([torch.arange(f, f + n, device="cuda") for n, f in zip(counts, first)])
        return pos.to(torch.int32), cu

    # all tokens at once ...
    pos, cu = places([n + more for n in lengths], [0] * len(lengths))
    all_at_once = layer(pack(-1, more), pos, cu)
    # ... and the prompts first, then one token of every sequence at a time
    cache = Cache(len(lengths), max(lengths) + more, Hk, D, torch.bfloat16, "cuda")
    pos, cu_p = places(lengths, [0] * len(lengths))
    layer.step(pack(-1, 0), pos, cu_p, cache)
    worst = 0.0
    for i in range(more):
        pos, one = places([1] * len(lengths), [n + i for n in lengths])
        y = layer.step(pack(i, i + 1), pos, one, cache).float()
        want = all_at_once[(cu[1:] - more + i).long()].float()
        worst = max(worst, float((y - want).norm() / want.norm()))
    print(f"prompts of {lengths} tokens, then {more} tokens each: token by token against all at once, "
          f"relative difference {worst:.1e}")


if __name__ == "__main__":
    main()
