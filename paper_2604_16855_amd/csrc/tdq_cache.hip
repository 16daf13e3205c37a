// A cache of keys and values in pages: new tokens written to it with norm and rotation on the way, the
// bounds of its pages, and the pages that a token attends to.
#include "tdq_pages.hpp"
#include "tdq_rotate.hpp"

namespace tdq {

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
// The arithmetic of the head norm (tdq_attention.hip) on the rows of a token's queries and keys; its
// values are copied.  A token is key len - n + i of its sequence (i of n new ones), which says where its
// keys and values go and, if no other is given, its position.  Every row is read and written once.  A
// workgroup takes a few whole tokens; a wavefront finds the place of each while the rows are on their
// way.
struct AppendArgs {
  const void* in[3];                   // Q, K, V
  long long in_token[3], in_head[3];
  void* out[3];                        // Qo, pages of K, pages of V
  long long out_token[3], out_head[3], page[3];
  const float* weight[2];
  int heads[3];                        // ends of the heads of Q, K and V in a token's row of all
  Sequences seq;
  long long T;
  int D, R, axes;
  float eps;
  const int* pos;                      // (nullptr: a token's place in its sequence)
  long long ld_pos;
  const int* axis;
  const float* freq;
};

constexpr int kAppendThreads = 256;
// Tokens of a workgroup in calls of many (one each in others); these leave rows behind each other that no
// cache holds until they are read, so their stores pass the caches by.  23052 tokens of 32/8 heads of 128,
// us: 1 token 121, 2 113, 4 117, 8-byte stores past the caches 108, with 2 tokens 105.
constexpr int kAppendTokens = 2, kAppendMany = 4096;

template <typename T, int L, bool PAIRS, bool MANY>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a) {
  constexpr int tokens = MANY ? kAppendTokens : 1;
  constexpr int GROUPS = kAppendThreads / L;           // heads at a time
  __shared__ float turn[kAppendTokens][TDQ_MAX_HEAD];  // cosine and sine of each pair
  __shared__ int place[kAppendTokens], page[kAppendTokens];   // key of its sequence, page (negative: nowhere, -2: no sequence)
  const int P = a.R >> 1;
  const long long t0 = (blockIdx.x + (long long)blockIdx.y * gridDim.x) * tokens;
  if (t0 >= a.T) return;                               // (a last row of workgroups may be longer than needed)
  const int here = (int)(a.T - t0 < tokens ? a.T - t0 : tokens);
  const int sub = threadIdx.x & (L - 1), first = threadIdx.x / L;
  const int D = a.D, R = a.R;
  const bool mine = 8 * sub < D, turned = 8 * sub < R;
  // 8 elements of a lane: neighbours, or 4 of the first half of the turned ones and their partners
  const int e0 = PAIRS || !turned ? 8 * sub : 4 * sub, e1 = PAIRS || !turned ? e0 + 4 : P + 4 * sub;
  struct Item {
    u32x2 a, b;
  };
  // Queries, keys or values of the workgroup's tokens: item i is head i % H of token i / H, the quotient
  // of small numbers by a reciprocal just above 1 / H.
  struct Kind {
    const T* in;
    T* out;
    long long in_token, in_head, out_token, out_head, page;
    const float* weight;
    int H;
    float per;
  };
  auto kind = [&](int which) {
    const int H = a.heads[which] - (which ? a.heads[which - 1] : 0);
    return Kind{static_cast<const T*>(a.in[which]) + t0 * a.in_token[which],
                static_cast<T*>(a.out[which]) + (which ? 0 : t0 * a.out_token[which]),
                a.in_token[which], a.in_head[which], a.out_token[which], a.out_head[which], a.page[which],
                which < 2 ? a.weight[which] : nullptr, H, 1.0f / (float)(H > 0 ? H : 1) * 1.000001f};
  };
  const Kind Q = kind(0), K = kind(1), V = kind(2);
  auto load = [&](const Kind& x, int i, Item& v) {
    const int t = (int)((float)i * x.per);
    const T* src = x.in + t * x.in_token + (i - t * x.H) * x.in_head;
    v.a = *reinterpret_cast<const u32x2_any*>(src + e0);
    v.b = *reinterpret_cast<const u32x2_any*>(src + e1);
  };
  auto load_all = [&](const Kind& x, int i, auto& v) {
#pragma unroll
    for (int u = 0; u < (int)(sizeof(v) / sizeof(v[0])); ++u)
      if (mine && i + u * GROUPS < here * x.H) load(x, i + u * GROUPS, v[u]);
  };
  // Many items are on their way while the places are found and the angles computed.
  Item q[4] = {}, k[2] = {}, v[2] = {};                 // (zeros where a head has nothing)
  load_all(Q, first, q);
  load_all(K, first, k);
  load_all(V, first, v);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave < here) {
    const Sequences& s = a.seq;
    const long long t = t0 + wave;
    const Owner o = owner_of(s, t, a.T);
    int j = -1, p = -2;
    if (t >= o.from && t < o.to) {
      j = (int)((long long)o.len - o.to + t);
      p = -1;
      if (o.len >= 0 && j >= 0 && j >> s.shift < s.columns) p = s.table[o.seq * s.ld + (j >> s.shift)];
      p = p >= 0 && p < s.n_pages ? p : -1;
    }
    if ((threadIdx.x & 63) == 0) {
      place[wave] = j;
      page[wave] = p;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < here * P; i += kAppendThreads) {
    const int t = i / P, p = i - t * P;
    int ax = a.axis ? a.axis[p] : 0;
    ax = ax < 0 ? 0 : ax < a.axes ? ax : a.axes - 1;
    const float angle = (float)(a.pos ? a.pos[ax * a.ld_pos + t0 + t] : place[t]) * a.freq[p];
    float s, c;
    turn_of(angle, &c, &s);
    turn[t][2 * p] = c;
    turn[t][2 * p + 1] = s;
  }
  __syncthreads();
  const int slots = (1 << a.seq.shift) - 1;
  // Where item i goes; nullptr: nowhere.
  auto place_of = [&](const Kind& x, bool cache, int i, int* token) -> T* {
    const int t = (int)((float)i * x.per), to = page[t];
    *token = t;
    if (to < (cache ? 0 : -1)) return nullptr;
    return x.out + (cache ? to * x.page + (place[t] & slots) * x.out_token : t * x.out_token) + (i - t * x.H) * x.out_head;
  };
  auto put = [&](T* p, u32x2 x) {
    if constexpr (MANY) __builtin_nontemporal_store(x, reinterpret_cast<u32x2_any*>(p));
    else *reinterpret_cast<u32x2_any*>(p) = x;
  };
  auto finish = [&](const Kind& x, bool cache, int i, const Item& v) {
    if (i >= here * x.H) return;                       // (the same in all lanes of a head)
    int t;
    T* dst = place_of(x, cache, i, &t);
    if (!dst) return;
    float f[4], g[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x2 y = two_floats<T>(v.a[j]), z = two_floats<T>(v.b[j]);
      f[2 * j] = y[0];
      f[2 * j + 1] = y[1];
      g[2 * j] = z[0];
      g[2 * j + 1] = z[1];
    }
    norm_and_turn<L, PAIRS>(f, g, x.weight, e0, e1, D, a.eps, mine, turned, &turn[t][8 * sub]);
    if (mine) {
      put(dst + e0, u32x2{two_rounded<T>(f[0], f[1]), two_rounded<T>(f[2], f[3])});
      put(dst + e1, u32x2{two_rounded<T>(g[0], g[1]), two_rounded<T>(g[2], g[3])});
    }
  };
  auto copy = [&](int i, const Item& x) {
    if (i >= here * V.H || !mine) return;
    int t;
    T* dst = place_of(V, true, i, &t);
    if (!dst) return;
    put(dst + e0, x.a);
    put(dst + e1, x.b);
  };
  for (int i = first; i < here * V.H; i += 2 * GROUPS) {
    if (i != first) load_all(V, i, v);
#pragma unroll
    for (int u = 0; u < 2; ++u) copy(i + u * GROUPS, v[u]);
  }
  for (int i = first; i < here * K.H; i += 2 * GROUPS) {
    if (i != first) load_all(K, i, k);
#pragma unroll
    for (int u = 0; u < 2; ++u) finish(K, true, i + u * GROUPS, k[u]);
  }
  for (int i = first; i < here * Q.H; i += 4 * GROUPS) {
    if (i != first) load_all(Q, i, q);
#pragma unroll
    for (int u = 0; u < 4; ++u) finish(Q, false, i + u * GROUPS, q[u]);
  }
}

hipError_t launch_append(const tdq_heads* Q, const tdq_heads* K, const tdq_heads* V, tdq_dtype dt, long long T,
                         const tdq_sequences* seq, int Hq, int Hk, int D, const float* q_weight, const float* k_weight,
                         float eps, int R, bool interleaved, const int* pos, long long ld_pos, int axes,
                         const int* axis, const float* freq, const tdq_heads* Qo, const tdq_pages* Kp,
                         const tdq_pages* Vp, hipStream_t st) {
  AppendArgs a;
  const tdq_heads none = {nullptr, 0, 0};
  const tdq_heads* in[3] = {Q ? Q : &none, K, V};
  for (int i = 0; i < 3; ++i) {
    a.in[i] = in[i]->data;
    a.in_token[i] = in[i]->token;
    a.in_head[i] = in[i]->head;
  }
  const tdq_heads* q = Qo ? Qo : &none;
  a.out[0] = q->data;
  a.out_token[0] = q->token;
  a.out_head[0] = q->head;
  a.page[0] = 0;
  const tdq_pages* out[2] = {Kp, Vp};
  for (int i = 0; i < 2; ++i) {
    a.out[i + 1] = out[i]->data;
    a.out_token[i + 1] = out[i]->token;
    a.out_head[i + 1] = out[i]->head;
    a.page[i + 1] = out[i]->page;
  }
  a.weight[0] = q_weight;
  a.weight[1] = k_weight;
  a.heads[0] = Hq;
  a.heads[1] = Hq + Hk;
  a.heads[2] = Hq + 2 * Hk;
  a.seq = sequences_of(seq);
  a.T = T;
  a.D = D;
  a.R = R;
  a.axes = axes;
  a.eps = eps;
  a.pos = pos;
  a.ld_pos = ld_pos;
  a.axis = axis;
  a.freq = freq;
  const int tokens = T >= kAppendMany ? kAppendTokens : 1;
  const dim3 grid = two_axes((T + tokens - 1) / tokens);
#define TDQ_APPEND_LP(T_, L, PAIRS)                                                                                \
  do {                                                                                                             \
    if (tokens > 1) hipLaunchKernelGGL((k_append<T_, L, PAIRS, true>), grid, dim3(kAppendThreads), 0, st, a);      \
    else hipLaunchKernelGGL((k_append<T_, L, PAIRS, false>), grid, dim3(kAppendThreads), 0, st, a);                \
  } while (0)
#define TDQ_APPEND_L(T_, L)                      \
  do {                                           \
    if (interleaved) TDQ_APPEND_LP(T_, L, true); \
    else TDQ_APPEND_LP(T_, L, false);            \
  } while (0)
#define TDQ_APPEND(T_)                         \
  do {                                         \
    if (D <= 32) TDQ_APPEND_L(T_, 4);          \
    else if (D <= 64) TDQ_APPEND_L(T_, 8);     \
    else if (D <= 128) TDQ_APPEND_L(T_, 16);   \
    else TDQ_APPEND_L(T_, 32);                 \
  } while (0)
  if (dt == TDQ_F16) TDQ_APPEND(_Float16);
  else TDQ_APPEND(__bf16);
#undef TDQ_APPEND
#undef TDQ_APPEND_L
#undef TDQ_APPEND_LP
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// bounds of pages
// ---------------------------------------------------------------------------
// Smallest and largest value of every channel over the keys of a page that are in use; NaN where one
// is.  A workgroup has a page and a key head: a lane 8 channels of every 16th row or so (all of them on
// their way at once), joined in the wavefront by exchanges and between wavefronts in LDS.  Bound by memory where
// there are many pages (48 MB in 11 us, 4.4 TB/s), and by three loads that wait for each other where there are
// few: 64 pages 6 us.
struct BoundsArgs {
  const void* K;
  void *lo, *hi;
  long long k_page, k_token, k_head, lo_page, lo_head, hi_page, hi_head;
  Sequences seq;
  long long T, slots;
  int Hk, D;
};

// (minimum and maximum that are NaN where one of the two is)
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <typename T, int L>
__global__ __launch_bounds__(256) void k_bounds(BoundsArgs a) {
  constexpr int GROUPS = 256 / L;                      // rows at a time
  __shared__ float part[3][2][8 * L];
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int h = (int)(id % a.Hk);
  const long long slot = id / a.Hk;
  if (slot >= a.slots) return;
  const Sequences& q = a.seq;
  int s, b;                                            // sequence and page of it
  if (q.cu) {
    // n new tokens lie in no more than n / P + 2 pages: sequence s has the slots from
    // floor(first token / P) + 2 s on
    s = last_at_most(q.S, slot, [&](int i) { return (long long)(start_of(q.cu, i, a.T) >> q.shift) + 2ll * i; });
    const int from = start_of(q.cu, s, a.T), n = start_of(q.cu, s + 1, a.T) - from, len = q.len[s];
    if (n <= 0) return;
    const long long i = slot - ((from >> q.shift) + 2ll * s);
    if (i < 0 || i >= q.columns) return;
    b = (int)i + ((len > n ? len - n : 0) >> q.shift);
  } else {
    s = (int)(slot / q.columns);
    b = (int)(slot - (long long)s * q.columns);
  }
  const int len = keys_of(q, s);
  if (b >= q.columns || b << q.shift >= len) return;
  const int page = q.table[s * q.ld + b];
  if (page < 0 || page >= q.n_pages) return;
  const int rest = len - (b << q.shift), rows = rest < 1 << q.shift ? rest : 1 << q.shift;
  const int sub = threadIdx.x & (L - 1), group = threadIdx.x / L, wave = threadIdx.x >> 6;
  const bool mine = 8 * sub < a.D;
  float lo[8], hi[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo[j] = INFINITY;
    hi[j] = -INFINITY;
  }
  const T* src = static_cast<const T*>(a.K) + page * a.k_page + h * a.k_head + 8 * sub;
  if (mine) {
#pragma unroll 4
    for (int r = group; r < rows; r += GROUPS) {
      float x[8];
      load_floats<T, 8>(src + r * a.k_token, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        lo[j] = least(lo[j], x[j]);
        hi[j] = most(hi[j], x[j]);
      }
    }
  }
#pragma unroll
  for (int d = L; d < 64; d <<= 1)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      lo[j] = least(lo[j], __shfl_xor(lo[j], d, 64));
      hi[j] = most(hi[j], __shfl_xor(hi[j], d, 64));
    }
  if (wave > 0 && (threadIdx.x & 63) < L) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      part[wave - 1][0][8 * sub + j] = lo[j];
      part[wave - 1][1][8 * sub + j] = hi[j];
    }
  }
  __syncthreads();
  if (threadIdx.x < L && mine) {
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        lo[j] = least(lo[j], part[w][0][8 * sub + j]);
        hi[j] = most(hi[j], part[w][1][8 * sub + j]);
      }
    store_floats<T, 8>(static_cast<T*>(a.lo) + page * a.lo_page + h * a.lo_head + 8 * sub, lo);
    store_floats<T, 8>(static_cast<T*>(a.hi) + page * a.hi_page + h * a.hi_head + 8 * sub, hi);
  }
}

hipError_t launch_bounds(const tdq_pages* K, tdq_dtype dt, long long T, const tdq_sequences* seq, int Hk, int D,
                         const tdq_heads* lo, const tdq_heads* hi, hipStream_t st) {
  BoundsArgs a;
  a.K = K->data;
  a.k_page = K->page;
  a.k_token = K->token;
  a.k_head = K->head;
  a.lo = lo->data;
  a.lo_page = lo->token;
  a.lo_head = lo->head;
  a.hi = hi->data;
  a.hi_page = hi->token;
  a.hi_head = hi->head;
  a.seq = sequences_of(seq);
  a.T = T;
  a.slots = a.seq.cu ? (T >> a.seq.shift) + 2ll * a.seq.S : (long long)a.seq.S * a.seq.columns;
  a.Hk = Hk;
  a.D = D;
  const dim3 grid = two_axes(a.slots * Hk);
#define TDQ_BOUNDS(T_)                                                                      \
  do {                                                                                      \
    if (D <= 32) hipLaunchKernelGGL((k_bounds<T_, 4>), grid, dim3(256), 0, st, a);          \
    else if (D <= 64) hipLaunchKernelGGL((k_bounds<T_, 8>), grid, dim3(256), 0, st, a);     \
    else if (D <= 128) hipLaunchKernelGGL((k_bounds<T_, 16>), grid, dim3(256), 0, st, a);   \
    else hipLaunchKernelGGL((k_bounds<T_, 32>), grid, dim3(256), 0, st, a);                 \
  } while (0)
  if (dt == TDQ_F16) TDQ_BOUNDS(_Float16);
  else TDQ_BOUNDS(__bf16);
#undef TDQ_BOUNDS
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// choice of pages
// ---------------------------------------------------------------------------
//   score[t, h, b] = max over the query heads e of h of sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d
// with q = Q[t, e] and the bounds of page b: no product of q with a key of the page is larger.
// The choice depends on which of two scores is larger, so they must not depend on the order of the sum:
// products of two 16-bit types are added in binary64, which holds nearly all such sums without rounding,
// and the result is rounded to binary32.  The products are the 64-bit matrix instruction's: 16 pages x 4
// heads x 4 channels at a time, four heads of a group and both of their signs in registers for all pages
// of a workgroup.  What bounds it is the way to the first bounds (the token's sequence, its pages, the
// bounds: 4 us), and beside the products the conversions of both operands: 32 tokens over 560 pages each, 8
// heads of 128, 26 us (73 MB).  By products in binary32 with a bound of their error, and in binary64 only
// where the order stays open, the scores took 21, but the choice 19 instead of 8.
// Which kernels run, and on how many workgroups, follows the width of the table, as the host does not know the
// lengths.  us with tables of no more columns than pages, of 1025 and of 8192: 32 tokens over 134 to 1001 pages:
// 34, 34 and 48; 401 over up to 508: 34, 45 and 213; 2000 over 141: 168, 339 and 1240; 8745 over up to 423: 108, 241
// and 2088.
struct ChoiceArgs {
  const void *Q, *lo, *hi;
  long long q_token, q_head, lo_page, lo_head, hi_page, hi_head;
  Sequences seq;
  long long Tq;
  int Hk, group, D, causal, first, last, count, chunks;
  float* score;                        // [Tq Hk, columns]
  int* chosen;                         // [Tq Hk, count]
};

// The sequence of a token and how many keys it sees (none: a token of no sequence).
struct Seen {
  int seq, keys;
};
__device__ __forceinline__ Seen seen_by(const Sequences& q, long long t, long long T, int causal) {
  const Owner o = owner_of(q, t, T);
  if (t < o.from || t >= o.to) return {o.seq, -1};
  return {o.seq, keys_seen(q, o.len, o.to, t, causal)};
}

// The value of lane ^ 1 or lane ^ 2.
template <int D>
__device__ __forceinline__ float neighbour(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), D == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true));
}

// Scores as they stand in an order of whole numbers: 0 is a page that is not there, the largest one that is
// always taken, NaN above all numbers.
constexpr u32 kAlways = 0xFFFFFFFFu, kNaN = 0xFFFFFFFEu;
__device__ __forceinline__ u32 key_of(float s) {
  if (s != s) return kNaN;
  const u32 u = __float_as_uint(s + 0.f);                // (-0 as 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The pages of a token and key head: a radix select of the count-th largest key among the scores'
// bit patterns (8 bits a pass), then the pages above it and the first ones at it, ascending.  Keys of
// 256 HELD pages stay in registers, and `entry` is what the line of the table has of them.  Bound by the
// passes' barriers, one after the other: 8 us for 256 lists of 560 pages on average; behind the scores in one
// kernel, 401 tokens' calls are shorter by 5 (39.7 to 34.9).
template <int HELD>
struct ChoiceRoom {
  u32 bins[256];
  u32 found[4];                                          // digit, keys of larger ones, keys of it
  u32 ends[2][4];
  int count[2][4 * HELD];                                // above the limit, and at it
};
template <int HELD, typename F>
__device__ __forceinline__ void choose(const ChoiceArgs& a, ChoiceRoom<HELD>& room, long long id, int pages, const int* line,
                                       const int (&entry)[HELD], F score) {
  auto &bins = room.bins;
  auto &found = room.found;
  auto &ends = room.ends;
  auto &count = room.count;
  int* out = a.chosen + id * a.count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto key = [&](int b, int page, float s) -> u32 {
    if (b >= pages || page < 0 || page >= a.seq.n_pages) return 0;
    return b < a.first || b >= pages - a.last ? kAlways : key_of(s);
  };
  auto read = [&](int b) { return b < pages ? key(b, line[b], score(b)) : 0; };
  u32 held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int b = 256 * i + tid;
    held[i] = key(b, entry[i], b < pages ? score(b) : 0.f);
  }
  auto each = [&](auto f) {                              // all pages, 256 at a time
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (256 * i < pages) f(256 * i + tid, held[i]);
    for (int b = 256 * HELD; b < pages; b += 256) f(b + tid, read(b + tid));
  };
  // Keys begin with the bits that all of them share but those at the two ends; the digits follow.
  u32 both = 0xFFFFFFFFu, any = 0;
  each([&](int, u32 k) {
    if (k != 0 && k < kNaN) {
      both &= k;
      any |= k;
    }
  });
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    both &= __shfl_xor(both, d, 64);
    any |= __shfl_xor(any, d, 64);
  }
  if (lane == 0) {
    ends[0][wave] = both;
    ends[1][wave] = any;
  }
  bins[tid] = 0;
  __syncthreads();
  u32 ands = 0xFFFFFFFFu, ors = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    ands &= ends[0][w];
    ors |= ends[1][w];
  }
  const bool some = ors != 0;
  u32 want = (u32)a.count, limit = 0;                    // taken: keys above limit, and the first `want` at it
  bool all = pages <= a.count, done = false;
  if (!all) {
    // those that are always taken, or NaN, come first: the lowest places of them if they are too many
    u32 c = 0;
    u32 top_keys = kAlways;
    for (int round = 0; round < 2 && !done; ++round, --top_keys) {
      c = 0;
      each([&](int, u32 k) { c += (u32)__popcll(__ballot(k == top_keys)); });
      if (lane == 0) found[wave] = c;
      __syncthreads();
      c = found[0] + found[1] + found[2] + found[3];
      __syncthreads();
      if (c >= want) {
        limit = top_keys;
        done = true;
      } else {
        want -= c;
      }
    }
    if (!done && !some) all = done = true;
  }
  const u32 differ = ands ^ ors;
  int bits = differ ? 32 - __builtin_clz(differ) : 0;    // low bits that are not the same in all
  u32 prefix = bits < 32 ? ands >> bits << bits : 0;
  if (!all && !done && bits == 0) limit = prefix;        // (one key, however often; fewer than wanted: all of them)
  while (!all && !done && bits > 0) {
    const int shift = bits > 8 ? bits - 8 : 0;
    each([&](int, u32 k) {
      if (k != 0 && k < kNaN && (bits == 32 || k >> bits == prefix >> bits)) atomicAdd(&bins[k >> shift & ((1u << (bits - shift)) - 1)], 1u);
    });
    __syncthreads();
    if (wave == 0) {
      u32 c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = bins[4 * lane + i];
        sum += c[i];
      }
      u32 upto = sum;                                    // of this lane's bins and all larger ones
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const u32 o = __shfl_down(upto, d, 64);
        if (lane + d < 64) upto += o;
      }
      u32 above = upto - sum;
      if (lane == 0 && upto < want) found[0] = 256;      // fewer keys than wanted: all of them
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        if (above < want && above + c[i] >= want) {
          found[0] = 4 * lane + i;
          found[1] = above;
          found[2] = c[i];
        }
        above += c[i];
      }
    }
    __syncthreads();
    bins[tid] = 0;
    if (found[0] == 256) {
      all = true;
    } else {
      prefix |= found[0] << shift;
      want -= found[1];
      limit = prefix;
      if (found[2] == want && shift > 0) {               // every key of the bin: nothing to tell apart
        all = prefix == 0;                               // (the lowest bin: every page that is there)
        limit = prefix - 1;
        want = 0;
        done = true;
      }
    }
    bits = shift;
    __syncthreads();
  }
  if (all) limit = 0;
  auto takes = [&](u32 k, bool* same) {
    *same = !all && k != 0 && k == limit && want > 0;
    return k > limit;
  };
  const unsigned long long below = (1ull << lane) - 1;
  // those in registers: counts of 256 at a time and wavefront, then a place for each
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    bool same;
    const bool more = takes(held[i], &same);
    const unsigned long long m = __ballot(more), e = __ballot(same);
    if (lane == 0) {
      count[0][4 * i + wave] = __popcll(m);
      count[1][4 * i + wave] = __popcll(e);
    }
  }
  __syncthreads();
  // sums over what stands in front: lane 4 i + w
  int mine_m = lane < 4 * HELD ? count[0][lane] : 0, mine_e = lane < 4 * HELD ? count[1][lane] : 0;
  int upto_m = mine_m, upto_e = mine_e;
#pragma unroll
  for (int d = 1; d < 4 * HELD; d <<= 1) {
    const int m = __shfl_up(upto_m, d, 64), e = __shfl_up(upto_e, d, 64);
    if (lane >= d) {
      upto_m += m;
      upto_e += e;
    }
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    bool same;
    const bool more = takes(held[i], &same);
    const unsigned long long m = __ballot(more), e = __ballot(same);
    const int at_m = __shfl(upto_m - mine_m, 4 * i + wave, 64), at_e = __shfl(upto_e - mine_e, 4 * i + wave, 64);
    const int rank = at_e + __popcll(e & below);         // among those at the limit
    // (of those at the limit in front, the first `want` are taken)
    const int before = at_m + __popcll(m & below) + (rank < (int)want ? rank : (int)want);
    if (more || (same && rank < (int)want)) out[before] = 256 * i + tid;
  }
  int taken_m = __shfl(upto_m, 4 * HELD - 1, 64), taken_e = __shfl(upto_e, 4 * HELD - 1, 64);
  for (int b = 256 * HELD; b < pages; b += 256) {
    bool same;
    const bool more = takes(read(b + tid), &same);
    const unsigned long long m = __ballot(more), e = __ballot(same);
    __syncthreads();
    if (lane == 0) {
      count[0][wave] = __popcll(m);
      count[1][wave] = __popcll(e);
    }
    __syncthreads();
    int at_m = taken_m, at_e = taken_e;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      at_m += w < wave ? count[0][w] : 0;
      at_e += w < wave ? count[1][w] : 0;
      taken_m += count[0][w];
      taken_e += count[1][w];
    }
    const int rank = at_e + __popcll(e & below);
    const int before = at_m + __popcll(m & below) + (rank < (int)want ? rank : (int)want);
    if (more || (same && rank < (int)want)) out[before] = b + tid;
  }
  const int taken = taken_m + (taken_e < (int)want ? taken_e : (int)want);
  for (int i = taken + tid; i < a.count; i += 256) out[i] = -1;
}

template <int HELD>
__device__ __forceinline__ void entries(const int* line, int pages, int (&entry)[HELD]) {
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int b = 256 * i + threadIdx.x;
    entry[i] = b < pages ? line[b] : -1;
  }
}

// The positive and the negative ones of 8 numbers, zeros in place of the others.
template <typename T>
__device__ __forceinline__ void signs_of(const u32x4& x, float* up, float* down) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 v = two_floats<T>(x[j]);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      up[2 * j + u] = v[u] < 0.f ? 0.f : v[u];
      down[2 * j + u] = v[u] > 0.f ? 0.f : v[u];
    }
  }
}

// Pages of a workgroup, 16 of a wavefront at a time.  us of both kernels with 256 and 512: D = 64, 401 tokens
// over 383 pages on average 47 and 35 (512 are all pages, and the choice is made here), 32 tokens over 469
// 18.5 and 16.2, 4 over 938 16 and 20; D = 128, 32 over 560 34 and 38, 4 over 938 22 and 30.
constexpr int score_pages(int W) { return W <= 16 ? 512 : 256; }

// W: channels of a lane.  Lane 16 k + p has of page p the 16-byte pieces k, k + 4, ..  WHOLE: a workgroup
// has all pages of a line, and makes the choice as well.
template <typename T, int W, bool WHOLE>
__global__ __launch_bounds__(256, W == 16 ? 3 : 4) void k_score(ChoiceArgs a) {
  constexpr int PIECES = W < 32 ? W / 8 : 4, PASSES = W / (8 * PIECES);   // pieces of a bound at a time
  constexpr int PAGES = score_pages(W);
  constexpr int HELD = PAGES / 256;
  __shared__ float top[PAGES];
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int h = (int)(id % a.Hk), chunk = (int)(id / a.Hk % a.chunks);
  const long long t = id / a.Hk / a.chunks;
  if (t >= a.Tq) return;
  const Sequences& q = a.seq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k = lane >> 4;
  auto at = [&](int pass, int i) { return 8 * (k + 4 * (pass * PIECES + i)); };   // first channel of a piece
  // operand columns: head lane % 4, its positive and its negative channels
  float up[8 * PIECES], down[8 * PIECES];
  auto query = [&](int e0, int pass) {
    // (past the last head: the last again, which changes no maximum)
    const int e = e0 + (lane & 3), head = h * a.group + (e < a.group ? e : a.group - 1);
    const T* p = static_cast<const T*>(a.Q) + t * a.q_token + head * a.q_head;
    u32x4 x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      x[i] = u32x4{0, 0, 0, 0};
      if (at(pass, i) < a.D) x[i] = *reinterpret_cast<const u32x4_any*>(p + at(pass, i));
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) signs_of<T>(x[i], up + 8 * i, down + 8 * i);
  };
  const Seen me = seen_by(q, t, a.Tq, a.causal);
  const int pages = me.keys <= 0 ? 0 : ((me.keys - 1) >> q.shift) + 1, b0 = chunk * PAGES;
  if (WHOLE ? me.keys < 0 : b0 + 16 * wave >= pages) return;
  const int here = pages - b0 < PAGES ? pages - b0 : PAGES;
  const int* line = q.table + me.seq * q.ld + b0;
  float* out = a.score + (t * a.Hk + h) * q.columns + b0;
  int entry[HELD];
  if constexpr (WHOLE) entries(line, pages, entry);
  // pages b .. b + 15: -1: none, or not there
  auto page_of = [&](int b) {
    int p = -1;
    if (b + (lane & 15) < here) p = line[b + (lane & 15)];
    return p < q.n_pages ? p : -1;
  };
#pragma unroll 1
  for (int e0 = 0; e0 < a.group; e0 += 4) {
    int page = page_of(16 * wave);
    if (PASSES == 1) query(e0, 0);
#pragma unroll 1
    for (int b = 16 * wave; b < here; b += 64) {
      const T* lo = static_cast<const T*>(a.lo) + (long long)page * a.lo_page + h * a.lo_head;
      const T* hi = static_cast<const T*>(a.hi) + (long long)page * a.hi_page + h * a.hi_head;
      double part[4] = {0.0, 0.0, 0.0, 0.0};             // (a product waits for the last one of its sum)
#pragma unroll 1
      for (int pass = 0; pass < PASSES; ++pass) {
        u32x4 los[PIECES], his[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          los[i] = his[i] = u32x4{0, 0, 0, 0};
          if (page >= 0 && at(pass, i) < a.D) {
            los[i] = *reinterpret_cast<const u32x4_any*>(lo + at(pass, i));
            his[i] = *reinterpret_cast<const u32x4_any*>(hi + at(pass, i));
          }
        }
        if (pass == PASSES - 1) page = page_of(b + 64);
        if (PASSES > 1) query(e0, pass);
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x2 l = two_floats<T>(los[i][j]), g = two_floats<T>(his[i][j]);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              // (converted again for every 16 pages: as binary64 they would take the registers of half of
              // the wavefronts that hide the bounds' way here)
              float x = up[8 * i + 2 * j + u], y = down[8 * i + 2 * j + u];
              if constexpr (W > 16) asm volatile("" : "+v"(x), "+v"(y));
              part[u] = __builtin_amdgcn_mfma_f64_4x4x4f64((double)g[u], (double)x, part[u], 0, 0, 0);
              part[2 + u] = __builtin_amdgcn_mfma_f64_4x4x4f64((double)l[u], (double)y, part[2 + u], 0, 0, 0);
            }
          }
      }
      // lane 16 i + 4 c + j has page 4 c + i and head j
      float best = (float)((part[0] + part[1]) + (part[2] + part[3]));
      best = most(best, neighbour<1>(best));
      best = most(best, neighbour<2>(best));
      const int mine = b + 4 * (lane >> 2 & 3) + (lane >> 4);
      if ((lane & 3) == 0 && mine < here) {              // (of pages that are not there nobody asks)
        if (e0 > 0) best = most(best, top[mine]);
        if (!WHOLE && e0 + 4 >= a.group) out[mine] = best;
        else top[mine] = best;                           // (up to here read by this lane alone)
      }
    }
  }
  if constexpr (WHOLE) {
    __shared__ ChoiceRoom<HELD> room;
    __syncthreads();
    choose(a, room, id, pages, line, entry, [&](int b) { return top[b]; });
  }
}

__global__ __launch_bounds__(256) void k_choose(ChoiceArgs a) {
  constexpr int HELD = 8;
  __shared__ ChoiceRoom<HELD> room;
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  if (id >= a.Tq * a.Hk) return;
  const Sequences& q = a.seq;
  const Seen me = seen_by(q, id / a.Hk, a.Tq, a.causal);
  if (me.keys < 0) return;                               // (no sequence: its pages are left as they are)
  const int pages = me.keys == 0 ? 0 : ((me.keys - 1) >> q.shift) + 1;
  const int* line = q.table + me.seq * q.ld;
  const float* score = a.score + id * q.columns;
  int entry[HELD];
  entries(line, pages, entry);
  choose(a, room, id, pages, line, entry, [&](int b) { return score[b]; });
}

// Many tokens of a sequence: 16 columns of tokens and 2^BITS heads at a time by the 16 x 16 x 4 instruction,
// so that the bounds are read, and converted, once for all of them.  A workgroup has TOKENS tokens and, where
// they are of several sequences, takes each run of them by itself; it keeps the keys of all their pages, and a
// wavefront makes the choice of a token without any other: the count-th largest key bit by bit, by ballots.
// Bound by that instruction (22 T products/s, two thirds of the small one's rate) and the ballots, about half
// each: 8745 tokens of 4/2 heads of 32 over 355 pages 102 us.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int kRunPages = 1024;        // of a line, at most
// Where it pays: two workgroups for every CU, and tokens of a sequence (on average, times the heads of a
// column) so that few workgroups have two runs, one after the other.  us by tokens on their own and by runs:
// 8745 tokens of 5 sequences, 4/2 heads of 32, over 355 pages 149 and 102; 2000 of 2, 32/8 of 128, over 142
// 224 and 169; 256 of one over 473 (512 workgroups) 101 and 66.  200 of one, 32/8 of 64, over 253 (400) 27 and
// 30; 128 of 4, 32/8 of 128, over 126 (256) 20 and 25.  30 times 30 tokens over 252 pages, 32/8 of 64 95 and
// 102, 8/8 of 128 164 and 102; 200 times 3, 16/4 of 128 69 and 101, 8/8 of 128 123 and 227.
constexpr long long kRunTokens = 16, kRunGroups = 512;
template <typename T, int W, int BITS>
__global__ __launch_bounds__(256, 2) void k_select_runs(ChoiceArgs a) {
  constexpr int PIECES = W < 32 ? W / 8 : 4, PASSES = W / (8 * PIECES);
  constexpr int TOKENS = 16 >> BITS, HEADS = 1 << BITS;
  __shared__ u32 keys[TOKENS][kRunPages];
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int h = (int)(id % a.Hk);
  const long long t0 = id / a.Hk * TOKENS;
  if (t0 >= a.Tq) return;
  const Sequences& q = a.seq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k = lane >> 4;
  const int token = (lane & 15) >> BITS, head = lane & (HEADS - 1);
  const unsigned long long below = (1ull << lane) - 1;
  auto at = [&](int pass, int i) { return 8 * (k + 4 * (pass * PIECES + i)); };   // first channel of a piece
  for (int first = 0, n; first < TOKENS && t0 + first < a.Tq; first += n) {
    const Owner o = owner_of(q, t0 + first, a.Tq);
    n = 1;
    if (t0 + first < o.from || t0 + first >= o.to) continue;
    n = o.to - t0 < TOKENS ? (int)(o.to - t0) - first : TOKENS - first;
    auto pages_of = [&](int i) {                         // that token first + i sees
      const int keys = keys_seen(q, o.len, o.to, t0 + first + i, a.causal);
      return keys == 0 ? 0 : ((keys - 1) >> q.shift) + 1;
    };
    const int pages = pages_of(n - 1);
    const int* line = q.table + o.seq * q.ld;
    const long long t = t0 + first + (token < n ? token : n - 1);   // of the lane's column
    auto page_of = [&](int b) {
      int p = -1;
      if (b + (lane & 15) < pages) p = line[b + (lane & 15)];
      return p < q.n_pages ? p : -1;
    };
#pragma unroll 1
    for (int e0 = 0; e0 < a.group; e0 += HEADS) {
      float up[8 * PIECES], down[8 * PIECES];
      auto query = [&](int pass) {
        // (past the last head: the last again, which changes no maximum)
        const int row = h * a.group + (e0 + head < a.group ? e0 + head : a.group - 1);
        const T* p = static_cast<const T*>(a.Q) + t * a.q_token + row * a.q_head;
        u32x4 x[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          x[i] = u32x4{0, 0, 0, 0};
          if (at(pass, i) < a.D) x[i] = *reinterpret_cast<const u32x4_any*>(p + at(pass, i));
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) signs_of<T>(x[i], up + 8 * i, down + 8 * i);
      };
      int page = page_of(16 * wave);
      if (PASSES == 1) query(0);
#pragma unroll 1
      for (int b = 16 * wave; b < pages; b += 64) {
        const T* lo = static_cast<const T*>(a.lo) + (long long)page * a.lo_page + h * a.lo_head;
        const T* hi = static_cast<const T*>(a.hi) + (long long)page * a.hi_page + h * a.hi_head;
        const unsigned there = (unsigned)__ballot(page >= 0);   // (of the first 16 lanes)
        f64x4 part[2] = {{0.0, 0.0, 0.0, 0.0}, {0.0, 0.0, 0.0, 0.0}};
#pragma unroll 1
        for (int pass = 0; pass < PASSES; ++pass) {
          u32x4 los[PIECES], his[PIECES];
#pragma unroll
          for (int i = 0; i < PIECES; ++i) {
            los[i] = his[i] = u32x4{0, 0, 0, 0};
            if (page >= 0 && at(pass, i) < a.D) {
              los[i] = *reinterpret_cast<const u32x4_any*>(lo + at(pass, i));
              his[i] = *reinterpret_cast<const u32x4_any*>(hi + at(pass, i));
            }
          }
          if (PASSES > 1) query(pass);
#pragma unroll
          for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const f32x2 l = two_floats<T>(los[i][j]), g = two_floats<T>(his[i][j]);
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                float x = up[8 * i + 2 * j + u], y = down[8 * i + 2 * j + u];
                if constexpr (W > 16) asm volatile("" : "+v"(x), "+v"(y));   // (as above)
                part[0] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)g[u], (double)x, part[0], 0, 0, 0);
                part[1] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)l[u], (double)y, part[1], 0, 0, 0);
              }
            }
        }
        page = page_of(b + 64);
        // element r of lane 16 i + j: page 4 r + i, column j
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float best = (float)(part[0][r] + part[1][r]);
          if (BITS > 0) best = most(best, neighbour<1>(best));
          if (BITS > 1) best = most(best, neighbour<2>(best));
          const int mine = 4 * r + k;
          if (head == 0 && b + mine < pages) {
            u32 x = there >> mine & 1 ? key_of(best) : 0;
            if (e0 > 0) x = max(x, keys[token][b + mine]);   // (written by this lane)
            keys[token][b + mine] = x;
          }
        }
      }
    }
    __syncthreads();
    for (int i = wave; i < n; i += 4) {
      const int seen = pages_of(i);
      int* out = a.chosen + ((t0 + first + i) * a.Hk + h) * a.count;
      u32 held[kRunPages / 64];
#pragma unroll
      for (int j = 0; j < kRunPages / 64; ++j) {
        const int b = 64 * j + lane;
        held[j] = 0;
        if (64 * j < seen) {
          if (b < seen) held[j] = keys[i][b];
          if (held[j] != 0 && (b < a.first || b >= seen - a.last)) held[j] = kAlways;
        }
      }
      // limit: the count-th largest, or 0 if there are fewer; `want` of those at it are taken
      u32 limit = 0;
      int want = 0;
      if (seen > a.count) {
        for (u32 bit = 1u << 31; bit; bit >>= 1) {
          const u32 at_least = limit | bit;
          int c = 0;
#pragma unroll
          for (int j = 0; j < kRunPages / 64; ++j)
            if (64 * j < seen) c += __popcll(__ballot(held[j] >= at_least));
          if (c < a.count) continue;
          limit = at_least;
          if (c == a.count) {                            // those and no others
            --limit;
            break;
          }
        }
        int above = 0;
#pragma unroll
        for (int j = 0; j < kRunPages / 64; ++j)
          if (64 * j < seen) above += __popcll(__ballot(held[j] > limit));
        want = limit > 0 ? a.count - above : 0;
      }
      int taken = 0, same = 0;                           // in front: above the limit, and at it
#pragma unroll
      for (int j = 0; j < kRunPages / 64; ++j)
        if (64 * j < seen) {
          const bool more = held[j] > limit, even = want > 0 && held[j] == limit;
          const unsigned long long m = __ballot(more), e = __ballot(even);
          const int rank = same + __popcll(e & below);
          const int place = taken + __popcll(m & below) + (rank < want ? rank : want);
          if (more || (even && rank < want)) out[place] = 64 * j + lane;
          taken += __popcll(m);
          same += __popcll(e);
        }
      taken += same < want ? same : want;
      for (int j = taken + lane; j < a.count; j += 64) out[j] = -1;
    }
    __syncthreads();                                     // (the keys have been read)
  }
}

size_t choice_workspace(long long Tq, int Hk, int columns) { return (size_t)Tq * Hk * columns * sizeof(float); }

hipError_t launch_choice(const tdq_heads* Q, const tdq_heads* lo, const tdq_heads* hi, tdq_dtype dt, long long Tq,
                         const tdq_sequences* seq, int Hq, int Hk, int D, bool causal, int first, int last, int count,
                         int* chosen, void* workspace, hipStream_t st) {
  ChoiceArgs a;
  a.Q = Q->data;
  a.q_token = Q->token;
  a.q_head = Q->head;
  a.lo = lo->data;
  a.lo_page = lo->token;
  a.lo_head = lo->head;
  a.hi = hi->data;
  a.hi_page = hi->token;
  a.hi_head = hi->head;
  a.seq = sequences_of(seq);
  a.Tq = Tq;
  a.Hk = Hk;
  a.group = Hq / Hk;
  a.D = D;
  a.causal = causal;
  a.first = first;
  a.last = last;
  a.count = count;
  a.score = static_cast<float*>(workspace);
  a.chosen = chosen;
  const int bits = a.group > 2 ? 2 : a.group - 1;
  const long long run_groups = (Tq + (16 >> bits) - 1) / (16 >> bits) * Hk;
  if (seq->columns <= kRunPages && Tq >= (kRunTokens << bits) * seq->S && run_groups >= kRunGroups) {
    const dim3 grid = two_axes(run_groups);
#define TDQ_RUN(T_, W)                                                                                    \
  do {                                                                                                    \
    if (bits == 2) hipLaunchKernelGGL((k_select_runs<T_, W, 2>), grid, dim3(256), 0, st, a);              \
    else if (bits == 1) hipLaunchKernelGGL((k_select_runs<T_, W, 1>), grid, dim3(256), 0, st, a);         \
    else hipLaunchKernelGGL((k_select_runs<T_, W, 0>), grid, dim3(256), 0, st, a);                        \
  } while (0)
#define TDQ_RUNS(T_)                    \
  do {                                  \
    if (D <= 32) TDQ_RUN(T_, 8);        \
    else if (D <= 64) TDQ_RUN(T_, 16);  \
    else if (D <= 128) TDQ_RUN(T_, 32); \
    else TDQ_RUN(T_, 64);               \
  } while (0)
    if (dt == TDQ_F16) TDQ_RUNS(_Float16);
    else TDQ_RUNS(__bf16);
#undef TDQ_RUNS
#undef TDQ_RUN
    return hipGetLastError();
  }
  const int pages = score_pages(D <= 32 ? 8 : D <= 64 ? 16 : D <= 128 ? 32 : 64);
  a.chunks = (seq->columns + pages - 1) / pages;
  const dim3 grid = two_axes(Tq * Hk * a.chunks);
#define TDQ_SCORE(T_, W)                                                                              \
  do {                                                                                                \
    if (a.chunks == 1) hipLaunchKernelGGL((k_score<T_, W, true>), grid, dim3(256), 0, st, a);         \
    else hipLaunchKernelGGL((k_score<T_, W, false>), grid, dim3(256), 0, st, a);                      \
  } while (0)
#define TDQ_SCORES(T_)                    \
  do {                                    \
    if (D <= 32) TDQ_SCORE(T_, 8);        \
    else if (D <= 64) TDQ_SCORE(T_, 16);  \
    else if (D <= 128) TDQ_SCORE(T_, 32); \
    else TDQ_SCORE(T_, 64);               \
  } while (0)
  if (dt == TDQ_F16) TDQ_SCORES(_Float16);
  else TDQ_SCORES(__bf16);
#undef TDQ_SCORES
#undef TDQ_SCORE
  if (a.chunks > 1) hipLaunchKernelGGL(k_choose, two_axes(Tq * Hk), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace tdq
