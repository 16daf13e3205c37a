// Sequences whose keys and values lie in the pages of a cache: what the kernels that write, sum up,
// choose and read pages share.
#pragma once

#include "tdq_half.hpp"

namespace tdq {

// tdq_sequences as the kernels take it.  Key j of sequence s is row j % P of page table[s][j / P].
struct Sequences {
  const int *cu, *len, *table;
  long long ld;
  int S, columns, n_pages, shift;      // page size P = 2^shift
};
inline Sequences sequences_of(const tdq_sequences* q) {
  Sequences s;
  s.cu = q->cu_q;
  s.len = q->len_k;
  s.table = q->table;
  s.ld = q->ld_table;
  s.S = q->S;
  s.columns = q->columns;
  s.n_pages = q->n_pages;
  s.shift = __builtin_ctz((unsigned)q->page_size);
  return s;
}

// cu[i] within 0 .. total.
__device__ __forceinline__ int start_of(const int* cu, long long i, long long total) {
  const int c = cu[i];
  return c < 0 ? 0 : c < total ? c : (int)total;
}
// Keys of a sequence: no more than its line of the table has room for.
__device__ __forceinline__ int keys_in(const Sequences& q, int len) {
  const int room = q.columns << q.shift;
  return len < 0 ? 0 : len < room ? len : room;
}
__device__ __forceinline__ int keys_of(const Sequences& q, int s) { return keys_in(q, q.len[s]); }
// Keys that token t sees of a sequence whose tokens end at `to`: it is key len - (to - t), also where that is
// past the room, and sees no key behind itself if causal.
__device__ __forceinline__ int keys_seen(const Sequences& q, int len, int to, long long t, bool causal) {
  const int n = keys_in(q, len);
  const long long e = (long long)len - to + t + 1;
  return !causal || e >= n ? n : e < 0 ? 0 : (int)e;
}

// The last i < n with first(i) <= at, for an ascending `first` with first(0) <= at: 64 places at a
// time, a lane each.  Every lane gets the answer.
template <typename F>
__device__ __forceinline__ int last_at_most(int n, long long at, F first) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 0) {
    const int step = (n + 63) / 64;
    const int i = lo + lane * step;
    const bool le = lane * step < n && first(i) <= at;
    const int count = __popcll(__ballot(le));            // (ascending: a run of lanes from 0 on)
    if (count == 0) break;
    const int base = lo + (count - 1) * step, rest = lo + n - base;
    lo = base;
    if (step == 1) break;
    n = rest < step ? rest : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The sequence of token t of T: which, its first token and the one behind its last (t is one of them, or
// of no sequence), and what stands in len.
struct Owner {
  int seq, from, to, len;
};
__device__ __forceinline__ Owner owner_of(const Sequences& q, long long t, long long T) {
  Owner o;
  if (q.S <= 64) {                                       // all at once, a lane each
    const int lane = threadIdx.x & 63, i = lane < q.S ? lane : q.S - 1;
    const int from = start_of(q.cu, i, T), to = start_of(q.cu, i + 1, T), len = q.len[i];
    const unsigned long long le = __ballot(lane < q.S && from <= t);
    o.seq = le ? 63 - __builtin_clzll(le) : 0;
    o.from = __builtin_amdgcn_readlane(from, o.seq);
    o.to = __builtin_amdgcn_readlane(to, o.seq);
    o.len = __builtin_amdgcn_readlane(len, o.seq);
  } else {
    o.seq = last_at_most(q.S, t, [&](int i) { return start_of(q.cu, i, T); });
    o.from = start_of(q.cu, o.seq, T);
    o.to = start_of(q.cu, o.seq + 1, T);
    o.len = q.len[o.seq];
  }
  return o;
}

}  // namespace tdq
