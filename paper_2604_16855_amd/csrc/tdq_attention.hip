// Norm of query and key heads with the rotation by position, and softmax attention with grouped
// heads over packed sequences.
#include <math.h>

#include "tdq_attend.hpp"
#include "tdq_rotate.hpp"

namespace tdq {

// ---------------------------------------------------------------------------
// norm and rotation
// ---------------------------------------------------------------------------
// y = x / sqrt(mean x^2 + eps) * w over a head's D elements, then pair p of the first R by the
// angle pos[axis of p] * freq[p]:  (a, b) -> (a cos - b sin, b cos + a sin).
// One pass: the rows are read and written once, bound by memory (32768 tokens of 32 heads of 64,
// binary16, in 60 us, 4.5 TB/s).  The angles of a token serve
// all its heads, so a workgroup takes a few whole tokens and leaves their cosines and sines in
// LDS.  The product pos * freq is rounded to binary32, as in the tables that models are trained
// with; from there on the angle is exact: it is reduced as a fraction of a turn in binary64.
struct RotateArgs {
  const void* in[2];
  void* out[2];
  const float* weight[2];
  long long in_token[2], in_head[2], out_token[2], out_head[2];
  int heads[2];
  long long T;
  int D, R, axes;
  float eps;
  const int* pos;
  long long ld_pos;
  const int* axis;
  const float* freq;
};

constexpr int kRotateThreads = 256;
constexpr int kMaxHead = 256;          // largest D
constexpr int kRotateTokens = 4;       // most tokens of a workgroup

template <typename T, int L, bool PAIRS>
__global__ __launch_bounds__(kRotateThreads) void k_norm_rotate(RotateArgs a, int tokens) {
  __shared__ float turn[kRotateTokens][kMaxHead];      // cosine and sine of each pair
  const int P = a.R >> 1;
  const long long t0 = (blockIdx.x + (long long)blockIdx.y * gridDim.x) * tokens;
  if (t0 >= a.T) return;                               // (a last row of workgroups may be longer than needed)
  const int here = (int)(a.T - t0 < tokens ? a.T - t0 : tokens);
  const int sub = threadIdx.x & (L - 1), heads = a.heads[0] + a.heads[1];
  const int D = a.D, R = a.R;
  const bool mine = 8 * sub < D, turned = 8 * sub < R;
  // 8 elements of a lane: neighbours, or 4 of the first half of the turned ones and their partners
  const int e0 = PAIRS || !turned ? 8 * sub : 4 * sub, e1 = PAIRS || !turned ? e0 + 4 : P + 4 * sub;
  // token and head of an item: the quotient of small numbers by a reciprocal just above 1 / heads
  const float per = 1.0f / (float)heads * 1.000001f;
  struct Item {
    float x[4], y[4];
  };
  auto load = [&](int i, Item& v) {
    const int t = (int)((float)i * per), hh = i - t * heads, which = hh >= a.heads[0], h = which ? hh - a.heads[0] : hh;
    const T* src = static_cast<const T*>(a.in[which]) + (t0 + t) * a.in_token[which] + h * a.in_head[which];
    load_floats<T, 4>(src + e0, v.x);
    load_floats<T, 4>(src + e1, v.y);
  };
  // The first items are on their way while the angles are computed, each next one while one is
  // worked on.
  const int first = threadIdx.x / L, items = here * heads;
  Item next = {};
  if (mine && first < items) load(first, next);
  for (int i = threadIdx.x; i < here * P; i += kRotateThreads) {
    const int t = i / P, p = i - t * P;
    int ax = a.axis ? a.axis[p] : 0;
    ax = ax < 0 ? 0 : ax < a.axes ? ax : a.axes - 1;
    const float angle = (float)a.pos[ax * a.ld_pos + t0 + t] * a.freq[p];
    float s, c;
    turn_of(angle, &c, &s);
    turn[t][2 * p] = c;
    turn[t][2 * p + 1] = s;
  }
  __syncthreads();
  for (int i = first; i < items; i += kRotateThreads / L) {
    Item v = next;
    if (mine && i + kRotateThreads / L < items) load(i + kRotateThreads / L, next);
    float(&x)[4] = v.x;
    float(&y)[4] = v.y;
    const int t = (int)((float)i * per), hh = i - t * heads, which = hh >= a.heads[0], h = which ? hh - a.heads[0] : hh;
    T* dst = static_cast<T*>(a.out[which]) + (t0 + t) * a.out_token[which] + h * a.out_head[which];
    norm_and_turn<L, PAIRS>(x, y, a.weight[which], e0, e1, D, a.eps, mine, turned, &turn[t][8 * sub]);
    if (mine) {
      store_floats<T, 4>(dst + e0, x);
      store_floats<T, 4>(dst + e1, y);
    }
  }
}

static RotateArgs rotate_args(const tdq_heads* Q, const tdq_heads* K, long long T, int Hq, int Hk, int D,
                              const float* q_weight, const float* k_weight, float eps, int R, const int* pos,
                              long long ld_pos, int axes, const int* axis, const float* freq, const tdq_heads* Qo,
                              const tdq_heads* Ko) {
  RotateArgs a;
  const tdq_heads none = {nullptr, 0, 0};
  const tdq_heads* in[2] = {Q, K ? K : &none};
  const tdq_heads* out[2] = {Qo, Ko ? Ko : &none};
  for (int i = 0; i < 2; ++i) {
    a.in[i] = in[i]->data;
    a.in_token[i] = in[i]->token;
    a.in_head[i] = in[i]->head;
    a.out[i] = out[i]->data;
    a.out_token[i] = out[i]->token;
    a.out_head[i] = out[i]->head;
  }
  a.weight[0] = q_weight;
  a.weight[1] = k_weight;
  a.heads[0] = Hq;
  a.heads[1] = Hk;
  a.T = T;
  a.D = D;
  a.R = R;
  a.axes = axes;
  a.eps = eps;
  a.pos = pos;
  a.ld_pos = ld_pos;
  a.axis = axis;
  a.freq = freq;
  return a;
}

hipError_t launch_norm_rotate(const tdq_heads* Q, const tdq_heads* K, tdq_dtype dt, long long T, int Hq, int Hk, int D,
                              const float* q_weight, const float* k_weight, float eps, int R, bool interleaved,
                              const int* pos, long long ld_pos, int axes, const int* axis, const float* freq,
                              const tdq_heads* Qo, const tdq_heads* Ko, hipStream_t st) {
  const RotateArgs a =
      rotate_args(Q, K, T, Hq, Hk, D, q_weight, k_weight, eps, R, pos, ld_pos, axes, axis, freq, Qo, Ko);
  const int tokens = T >= 1024 * kRotateTokens ? kRotateTokens : 1;
  const dim3 grid = two_axes((T + tokens - 1) / tokens);
#define TDQ_ROTATE_LP(T_, L, PAIRS) \
  hipLaunchKernelGGL((k_norm_rotate<T_, L, PAIRS>), grid, dim3(kRotateThreads), 0, st, a, tokens)
#define TDQ_ROTATE_L(T_, L)                    \
  do {                                         \
    if (interleaved) TDQ_ROTATE_LP(T_, L, true); \
    else TDQ_ROTATE_LP(T_, L, false);          \
  } while (0)
#define TDQ_ROTATE(T_)                         \
  do {                                         \
    if (D <= 32) TDQ_ROTATE_L(T_, 4);          \
    else if (D <= 64) TDQ_ROTATE_L(T_, 8);     \
    else if (D <= 128) TDQ_ROTATE_L(T_, 16);   \
    else TDQ_ROTATE_L(T_, 32);                 \
  } while (0)
  if (dt == TDQ_F16) TDQ_ROTATE(_Float16);
  else if (dt == TDQ_BF16) TDQ_ROTATE(__bf16);
  else TDQ_ROTATE(float);
#undef TDQ_ROTATE
#undef TDQ_ROTATE_L
#undef TDQ_ROTATE_LP
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
//   O[t, h] = sum_j softmax_j(scale q_t . k_j) v_j over the keys j of t's sequence that t sees.
// The query heads of a key head are rows of one tile: row r of a sequence is token r / g, head
// r % g of the group of g, so keys and values are read once for all of them, and one token
// (g rows) goes the same way as a prompt.  One pass over the keys with the running maximum and
// sum of the softmax (binary32); a wavefront has 32 rows:
//   S^T = K Q^T       keys x rows: a lane holds 16 of every 32 keys of ONE row, so that a row's
//                     maximum is 15 steps in the lane and one exchange of the two halves
//   P^T = 2^(c S^T - c m), rounded to the type of V as the matrix instruction's operand
//   O^T += V^T P^T    a lane's probabilities are its operand as they lie: the order of the keys
//                     within an instruction is free as long as V^T is read in the same order
// The maximum m that P refers to is raised, and O rescaled, only when a score exceeds it by 8
// octaves: the quotient O / sum is the same for any m, and 2^8 leaves every type its precision.
// Binary16 ends 25 octaves below 1, where many keys of a long cache may still have a weight together:
// its m is 7 octaves below the largest score, so that probabilities (at most 2^15) end 32 octaves
// below the largest.
// The sum of the probabilities is taken before their rounding.
struct AttendArgs {
  const void *Q, *K, *V;
  void* O;
  float* lse;
  const int *cu_q, *cu_k, *len_k;      // (len_k: nullptr, or how many of a sequence's keys are used)
  long long q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  long long Tq, Tk;
  int S, Hq, Hk, group, D, causal;
  float scale_log2;                    // |scale| log2(e), at least 1e-30 (a masked score stays -inf)
  float lift;                          // kLift octaves as a score
  u32 flip;                            // sign bits of two elements if the scale is negative: Q is negated
  int splits;                          // parts that the keys of a sequence are cut into
  float *part_o, *part_ml;             // [Tq Hq][splits][D], and maximum and sum [Tq Hq][splits][2]
};

// The sequence and the tile of a slot: sequence s has the slots from floor(first row / BM) + s
// on, which leaves it at least as many as it has tiles of BM rows.
struct Slot {
  int seq, tile;
};
__device__ __forceinline__ int clamp_start(const int* cu, int s, long long total) {
  const int c = cu[s];
  return c < 0 ? 0 : c < total ? c : (int)total;
}
template <int BM>
__device__ __forceinline__ Slot find_slot(const AttendArgs& a, long long slot) {
  // 64-way search for the last sequence whose first slot is not past this one
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.S;
  while (n > 0) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    bool le = false;
    if (lane * step < n) le = (long long)clamp_start(a.cu_q, at, a.Tq) * a.group / BM + at <= slot;
    const int count = __popcll(__ballot(le));          // (monotonic: a run of lanes from 0 on)
    if (count == 0) break;
    const int base = lo + (count - 1) * step;
    const int rest = lo + n - base;
    lo = base;
    if (step == 1) break;
    n = rest < step ? rest : step;
  }
  Slot r;
  r.seq = __builtin_amdgcn_readfirstlane(lo);
  r.tile = (int)(slot - ((long long)clamp_start(a.cu_q, r.seq, a.Tq) * a.group / BM + r.seq));
  r.tile = __builtin_amdgcn_readfirstlane(r.tile);
  return r;
}

// A tile of rows of a sequence.
struct Tile {
  int q0, nq, k0, nk;                  // first query and key of the sequence, and how many
  long long r0, rows;                  // first row of the tile, rows of the sequence
  int ahead;                           // a causal token t sees the keys up to t + ahead
  __device__ __forceinline__ bool none() const { return r0 < 0 || r0 >= rows; }
  // Keys that row r sees.
  __device__ __forceinline__ int sees(const AttendArgs& a, long long r) const {
    if (!a.causal) return nk;
    const long long e = r / a.group + ahead + 1;
    return e < 0 ? 0 : e < nk ? (int)e : nk;
  }
};
template <int BM>
__device__ __forceinline__ Tile find_tile(const AttendArgs& a, long long slot) {
  const Slot s = find_slot<BM>(a, slot);
  Tile t;
  t.q0 = clamp_start(a.cu_q, s.seq, a.Tq);
  t.nq = clamp_start(a.cu_q, s.seq + 1, a.Tq) - t.q0;
  t.k0 = clamp_start(a.cu_k, s.seq, a.Tk);
  t.nk = clamp_start(a.cu_k, s.seq + 1, a.Tk) - t.k0;
  if (a.len_k) {
    const int used = a.len_k[s.seq];
    t.nk = used < t.nk ? used : t.nk;
  }
  t.nk = t.nk > 0 ? t.nk : 0;
  t.rows = t.nq > 0 ? (long long)t.nq * a.group : 0;
  t.r0 = (long long)s.tile * BM;
  t.ahead = t.nk - t.nq;
  return t;
}

// One copy instruction: ROWS_PER_COPY rows of keys or values to LDS, zeros past the sequence's
// end and past D.
template <typename T, int DP, int PLACE(int)>
__device__ __forceinline__ void copy_rows(const T* first, long long token, int r, int left, int D, u32 lds) {
  constexpr int PIECES = DP / 8;
  const int lane = threadIdx.x & 63, row = r + lane / PIECES, piece = (lane % PIECES) ^ PLACE(row);
  const T* p = first + row * token + 8 * piece;
  copy_to_lds(row < left && 8 * piece < D ? (const void*)p : (const void*)kZeros, lds);
}

// The same for whole tiles, of N copies one after the other: offsets of this lane from the first
// row, so that a copy costs no vector instruction.
template <int DP, int N, int PLACE(int)>
struct CopyOffsets {
  u32 off[N];
  __device__ __forceinline__ CopyOffsets(long long token, int r) {
    constexpr int PIECES = DP / 8, ROWS = 64 / PIECES;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = r + i * ROWS + lane / PIECES;
      off[i] = (u32)(row * token * 2) + 16 * ((lane % PIECES) ^ PLACE(row));
    }
  }
  __device__ __forceinline__ void copy(const void* first, u32 lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) copy_to_lds(first, off[i], lds + 1024 * i);
  }
};
// Whether rows of a tile are within 32-bit offsets, and as long as in LDS.
__device__ __forceinline__ bool whole_rows(const AttendArgs& a, int DP) {
  return a.D == DP && a.k_token >= 0 && a.v_token >= 0 && a.k_token < 1 << 24 && a.v_token < 1 << 24;
}

constexpr int kKeys = 64;              // keys of a tile

// Many rows: 128 of them by four wavefronts that share tiles of 64 keys, the next tile on its way
// while one is worked on.  Bound by the matrix and the vector unit (45 and 53 % of the cycles, hardly
// at the same time): 8 causal prompts of up to 4096, 32/8 heads of 128, in 631 us, 930 TFLOP/s.
// With D up to 128 padded to a power of two (80 takes 586 us there, 96 605, at 620 and 730 TFLOP/s
// of what they need); beyond, tiles have one stage and a SIMD one wavefront: 16/4 heads of 256 865 us,
// 680 TFLOP/s.
template <typename T, int DP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 2 : 1))) void k_attend(AttendArgs a,
                                                                                               long long slots) {
  constexpr int BM = 128, ROW = DP * 2;                // bytes of a row in LDS
  constexpr int ROWS_PER_COPY = 512 / DP, COPIES = kKeys / ROWS_PER_COPY / 4;   // per wavefront
  constexpr int STAGES = DP <= 128 ? 2 : 1;
  __shared__ __attribute__((aligned(1024))) uint8_t kv[STAGES][2][kKeys * ROW];

  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  if (id >= slots * a.Hk) return;
  const int hk = (int)(id % a.Hk);
  const Tile t = find_tile<BM>(a, slots - 1 - id / a.Hk);
  if (t.none()) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, D = a.D;

  const long long first = t.r0 + wave * 32, row = first + (lane & 31);
  const bool real = row < t.rows;
  const long long row_c = real ? row : t.rows - 1;
  const int token = (int)(row_c / a.group), head = hk * a.group + (int)(row_c - (long long)token * a.group);
  const int sees = t.sees(a, row_c);
  // how many keys the workgroup needs, and all rows of this wavefront see
  const int end = __builtin_amdgcn_readfirstlane(t.sees(a, t.r0 + BM < t.rows ? t.r0 + BM - 1 : t.rows - 1));
  const int last = __builtin_amdgcn_readfirstlane(t.sees(a, first + 32 < t.rows ? first + 31 : t.rows - 1));
  const int all = __builtin_amdgcn_readfirstlane(t.sees(a, first < t.rows ? first : t.rows - 1));

  Rows<T, DP> w;
  w.start(static_cast<const T*>(a.Q) + (t.q0 + token) * a.q_token + head * a.q_head, D, a.flip);
  const T* kp = static_cast<const T*>(a.K) + t.k0 * a.k_token + hk * a.k_head;
  const T* vp = static_cast<const T*>(a.V) + t.k0 * a.v_token + hk * a.v_head;
  const bool quick = whole_rows(a, DP);
  const CopyOffsets<DP, COPIES, place_k<DP>> ko(a.k_token, wave * COPIES * ROWS_PER_COPY);
  const CopyOffsets<DP, COPIES, place_v<DP>> vo(a.v_token, wave * COPIES * ROWS_PER_COPY);
  auto copy_tile = [&](int j0, int stage) {
    const u32 lk = lds_address(kv[stage][0]), lv = lds_address(kv[stage][1]);
    const T *kt = kp + j0 * a.k_token, *vt = vp + j0 * a.v_token;
    if (quick && j0 + kKeys <= t.nk) {
      ko.copy(kt, lk + wave * COPIES * 1024);
      vo.copy(vt, lv + wave * COPIES * 1024);
      return;
    }
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const int c = wave * COPIES + i, r = c * ROWS_PER_COPY;
      copy_rows<T, DP, place_k<DP>>(kt, a.k_token, r, t.nk - j0, D, lk + c * 1024);
      copy_rows<T, DP, place_v<DP>>(vt, a.v_token, r, t.nk - j0, D, lv + c * 1024);
    }
  };
  w.addresses(lds_address(kv[0][0]), lds_address(kv[0][1]));
  if (STAGES == 2 && end > 0) copy_tile(0, 0);
  for (int j0 = 0; j0 < end; j0 += kKeys) {
    const int stage = STAGES == 2 ? (j0 / kKeys) & 1 : 0;
    if (STAGES == 1) {
      __syncthreads();                                 // the last tile has been read
      copy_tile(j0, 0);
    }
    wait_copies();
    __syncthreads();
    if (STAGES == 2 && j0 + kKeys < end) copy_tile(j0 + kKeys, stage ^ 1);
    if (j0 < last) {
      f32x16 s[2];
      u32 p[2][8];
      s[0] = w.scores(0);
      s[1] = w.scores(32);
      w.softmax(s, p, a.scale_log2, a.lift, j0 + kKeys > all, [&](int k) { return j0 + k < sees; });
      w.values(0, p[0]);
      w.values(32, p[1]);
    }
    if (STAGES == 2) w.move(stage ? -(int)sizeof(kv[0]) : (int)sizeof(kv[0]));
  }

  const float l = w.l + other_half(w.l);
  if (!real) return;
  // a row that sees no key: zeros, and -inf (its sums may hold 0 * NaN from values that others see)
  const bool none = no_weight(w.m, l);
  if (__ballot(none)) {                                // (hardly ever: no select in the ordinary way)
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) w.o[i][j] = none ? 0.f : w.o[i][j];
  }
  const float inv = none ? 0.f : 1.0f / l;
  T* op = static_cast<T*>(a.O) + (t.q0 + token) * a.o_token + head * a.o_head;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      const int c = 32 * i + 2 * j + 4 * half;
      if (c < D) {
        const float y[4] = {w.o[i][j] * inv, w.o[i][j + 1] * inv, w.o[i][j + 2] * inv, w.o[i][j + 3] * inv};
        store_floats<T, 4>(op + c, y);
      }
    }
  if (a.lse && half == 0) a.lse[(t.q0 + (long long)token) * a.Hq + head] = log_sum(w.m, l, a.scale_log2);
}

// Few rows (single tokens over a cache): 32 of them, and it is the keys that are shared out, to
// `splits` workgroups and in each to four wavefronts.  Bound by reading K and V once: a wavefront
// copies its own tiles of 32 keys, K of the next while it works on V of this and the other way
// round, and waits for nobody until the end, where the wavefronts' parts are joined in LDS.  16 tokens
// over 4000 to 32000 keys, 32/8 heads of 128: 222 us, 5.3 TB/s (a wavefront of rows for all keys: 1354);
// 16/4 heads of 256, with 17 registers in scratch, 3.1 TB/s.
constexpr int kFewRows = 32, kFewKeys = 32;
template <int DP>
struct FewShared {
  union {
    uint8_t kv[4][2][kFewKeys * 2 * DP];               // [wavefront][K, V]
    float o[4][32][DP + 4];                            // parts of the output, rows 16 bytes apart in the banks
  };
  float ml[4][32][2];
};

template <typename T, int DP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP <= 128 ? 2 : 1))) void k_attend_few(
    AttendArgs a, long long slots) {
  constexpr int ROWS_PER_COPY = 512 / DP, COPIES = kFewKeys / ROWS_PER_COPY;
  __shared__ __attribute__((aligned(1024))) FewShared<DP> sh;

  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int hk = (int)(id % a.Hk), split = (int)(id / a.Hk % a.splits);
  const long long slot = id / a.Hk / a.splits;
  if (slot >= slots) return;
  const Tile t = find_tile<kFewRows>(a, slots - 1 - slot);
  if (t.none()) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int D = a.D;
  const long long row = t.r0 + (lane & 31);
  const long long row_c = row < t.rows ? row : t.rows - 1;
  const int token = (int)(row_c / a.group), head = hk * a.group + (int)(row_c - (long long)token * a.group);
  const int sees = t.sees(a, row_c);
  const int here = (int)(t.rows - t.r0 < kFewRows ? t.rows - t.r0 : kFewRows);       // rows of the tile
  const int end = __builtin_amdgcn_readfirstlane(t.sees(a, t.r0 + here - 1));
  const int all = __builtin_amdgcn_readfirstlane(t.sees(a, t.r0));
  const int tiles = (end + kFewKeys - 1) / kFewKeys, share = (tiles + a.splits - 1) / a.splits;
  const int stop = (split + 1) * share < tiles ? (split + 1) * share : tiles;

  Rows<T, DP> w;
  w.template start<false>(static_cast<const T*>(a.Q) + (t.q0 + token) * a.q_token + head * a.q_head, D, a.flip);
  const T* kp = static_cast<const T*>(a.K) + t.k0 * a.k_token + hk * a.k_head;
  const T* vp = static_cast<const T*>(a.V) + t.k0 * a.v_token + hk * a.v_head;
  const u32 lk = lds_address(sh.kv[wave][0]), lv = lds_address(sh.kv[wave][1]);
  const bool quick = whole_rows(a, DP);
  const CopyOffsets<DP, COPIES, place_k<DP>> ko(a.k_token, 0);
  const CopyOffsets<DP, COPIES, place_v<DP>> vo(a.v_token, 0);
  auto copy_k = [&](int i) {
    const T* kt = kp + (long long)i * kFewKeys * a.k_token;
    if (quick && (i + 1) * kFewKeys <= t.nk) return ko.copy(kt, lk);
#pragma unroll
    for (int c = 0; c < COPIES; ++c)
      copy_rows<T, DP, place_k<DP>>(kt, a.k_token, c * ROWS_PER_COPY, t.nk - i * kFewKeys, D, lk + c * 1024);
  };
  auto copy_v = [&](int i) {
    const T* vt = vp + (long long)i * kFewKeys * a.v_token;
    if (quick && (i + 1) * kFewKeys <= t.nk) return vo.copy(vt, lv);
#pragma unroll
    for (int c = 0; c < COPIES; ++c)
      copy_rows<T, DP, place_v<DP>>(vt, a.v_token, c * ROWS_PER_COPY, t.nk - i * kFewKeys, D, lv + c * 1024);
  };
  w.addresses(lk, lv);
  int i = split * share + wave;
  if (i < stop) {
    copy_k(i);
    copy_v(i);
  }
  for (; i < stop; i += 4) {
    const bool more = i + 4 < stop;
    // (copies arrive in order: all but the last COPIES, those of V, are there)
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
    f32x16 s[1];
    u32 p[1][8];
    s[0] = w.scores(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K has been read
    if (more) copy_k(i + 4);
    w.softmax(s, p, a.scale_log2, a.lift, (i + 1) * kFewKeys > all,
              [&](int k) { return i * kFewKeys + k < sees; });
    if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
    else wait_copies();
    w.values(0, p[0]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V has been read
    if (more) copy_v(i + 4);
  }

  // join the wavefronts' parts: they refer to different maxima
  const float l = w.l + other_half(w.l);
  if (lane < 32) {
    sh.ml[wave][lane][0] = w.m;
    sh.ml[wave][lane][1] = l;
  }
  __syncthreads();                                       // (nobody reads K and V any more)
  float m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int v = 0; v < 4; ++v) m = fmaxf(m, sh.ml[v][lane & 31][0]);
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float mv = sh.ml[v][lane & 31][0], lv = sh.ml[v][lane & 31][1];
    if (!no_weight(mv, lv)) sum += lv * __builtin_amdgcn_exp2f((mv - m) * a.scale_log2);
  }
  // (a part in which a row sees no key is 0: its sums may hold 0 * NaN from values that others see)
  const bool none = no_weight(w.m, l);
  const float keep = __builtin_amdgcn_exp2f((w.m - m) * a.scale_log2);
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      f32x4 y;
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = none ? 0.f : w.o[d][j + u] * keep;
      *reinterpret_cast<f32x4*>(&sh.o[wave][lane & 31][32 * d + 2 * j + 4 * (lane >> 5)]) = y;
    }
  __syncthreads();
  if (wave == 0 && lane < 32) {                          // for the threads that store a row
    sh.ml[0][lane][0] = m;
    sh.ml[0][lane][1] = sum;
  }
  __syncthreads();
  constexpr int QUADS = DP / 4;
  for (int e = threadIdx.x; e < here * QUADS; e += 256) {
    const int r = e / QUADS, c = 4 * (e % QUADS);
    if (c >= D) continue;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 4; ++v) y += *reinterpret_cast<const f32x4*>(&sh.o[v][r][c]);
    const float mr = sh.ml[0][r][0], lr = sh.ml[0][r][1];
    const long long rr = t.r0 + r;
    const int tok = (int)(rr / a.group), h = hk * a.group + (int)(rr - (long long)tok * a.group);
    const long long at = (t.q0 + (long long)tok) * a.Hq + h;
    if (a.splits > 1) {
      const long long part = at * a.splits + split;
      *reinterpret_cast<f32x4*>(a.part_o + part * D + c) = y;
      if (c == 0) {
        a.part_ml[2 * part] = mr;
        a.part_ml[2 * part + 1] = lr;
      }
    } else {
      const float inv = no_weight(mr, lr) ? 0.f : 1.0f / lr;
      const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
      store_floats<T, 4>(static_cast<T*>(a.O) + (t.q0 + tok) * a.o_token + h * a.o_head + c, z);
      if (a.lse && c == 0) a.lse[at] = log_sum(mr, lr, a.scale_log2);
    }
  }
}

// Joins the splits' parts, a wavefront a row: its lanes take four outputs each of 256 / D' parts at a
// time (D' the next power of two), their weights found before, so that all parts are on their way
// at once.
constexpr int kMaxSplits = 128;
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, long long slots) {
  __shared__ float weight[4][kMaxSplits];
  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  if (id >= slots * a.Hk) return;
  const int hk = (int)(id % a.Hk);
  const Tile t = find_tile<kFewRows>(a, id / a.Hk);
  if (t.none()) return;
  const int here = (int)(t.rows - t.r0 < kFewRows ? t.rows - t.r0 : kFewRows);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int quads = a.D <= 32 ? 8 : a.D <= 64 ? 16 : a.D <= 128 ? 32 : 64;
  const int c = 4 * (lane & (quads - 1)), group = lane / quads, groups = 64 / quads;
  for (int r = wave; r < here; r += 4) {
    const long long rr = t.r0 + r;
    const int tok = (int)(rr / a.group), h = hk * a.group + (int)(rr - (long long)tok * a.group);
    const long long at = (t.q0 + (long long)tok) * a.Hq + h;
    const float* ml = a.part_ml + 2 * at * a.splits;
    float ms[kMaxSplits / 64], ls[kMaxSplits / 64], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxSplits / 64; ++i) {
      const int s = lane + 64 * i;
      ms[i] = s < a.splits ? ml[2 * s] : -INFINITY;
      ls[i] = s < a.splits ? ml[2 * s + 1] : 0.f;
      m = fmaxf(m, ms[i]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
#pragma unroll
    for (int i = 0; i < kMaxSplits / 64; ++i) {
      const int s = lane + 64 * i;
      // A part without keys is left out, marked by a negative weight.  One of nothing but NaN has the
      // same maximum of -inf, and its sum makes the row NaN; one whose weight rounds to 0 still counts,
      // as its values may not be finite.
      const bool none = no_weight(ms[i], ls[i]);
      const float f = ls[i] != ls[i] ? ls[i] : __builtin_amdgcn_exp2f((ms[i] - m) * a.scale_log2);
      if (s < a.splits) {
        weight[wave][s] = none ? -1.f : f;
        if (!none) l = fmaf(ls[i], f, l);
      }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d, 64);
    __builtin_amdgcn_wave_barrier();
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (c < a.D) {
      const float* po = a.part_o + at * a.splits * a.D + c;
#pragma unroll 8
      for (int s = group; s < a.splits; s += groups) {
        const float f = weight[wave][s];
        if (!(f < 0.f)) y += *reinterpret_cast<const f32x4*>(po + (long long)s * a.D) * f;
      }
    }
    for (int d = 32; d >= quads; d >>= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] += __shfl_xor(y[i], d, 64);
    const float inv = no_weight(m, l) ? 0.f : 1.0f / l;
    if (group == 0 && c < a.D) {
      const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
      store_floats<T, 4>(static_cast<T*>(a.O) + (t.q0 + tok) * a.o_token + h * a.o_head + c, z);
      if (a.lse && lane == 0)
        a.lse[at] = log_sum(m, l, a.scale_log2);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Which way a call goes, from what the host knows of it: the totals, not the sequences.  Keys are
// shared out where there are up to 32 rows a sequence on average, by the average of its keys.  Beyond
// that a workgroup goes through all keys of its 128 rows, which leaves most of the chip idle where
// there are few such tiles: one sequence over 30000 keys, 32/8 heads of 128, 8 tokens 192 us (160 of
// it the join, which has one workgroup for the rows of a tile), 9 tokens 534; 15 single tokens over 32000 keys 366 us, and 631 with a prompt of 2000 (54) in the same call.
struct AttendPlan {
  bool few;
  int splits;
};
static AttendPlan attend_plan(long long Tq, long long Tk, int S, int Hq, int Hk) {
  AttendPlan p = {false, 1};
  const long long g = Hq / Hk;
  if (Tq * g > 32ll * S) return p;
  p.few = true;
  // enough workgroups for 512 at a time to even out sequences of different lengths, as long as
  // each has a few hundred keys
  const long long most = Tk / S / 256, base = (long long)S * Hk;
  long long n = 2048 / base;
  if (n > most) n = most;
  if (n > kMaxSplits) n = kMaxSplits;
  if (n > 1) p.splits = (int)n;
  return p;
}

static size_t part_ml_bytes(long long Tq, int Hq, int splits) {
  return ((size_t)Tq * Hq * splits * 2 * sizeof(float) + 255) & ~(size_t)255;
}

size_t attention_workspace(long long Tq, long long Tk, int S, int Hq, int Hk, int D) {
  const AttendPlan p = attend_plan(Tq, Tk, S, Hq, Hk);
  if (p.splits <= 1) return 0;
  return part_ml_bytes(Tq, Hq, p.splits) + (size_t)Tq * Hq * p.splits * D * sizeof(float);
}

template <typename T, int DP>
static void launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (p.few) {
    const long long slots = a.Tq * a.group / kFewRows + a.S;
    hipLaunchKernelGGL((k_attend_few<T, DP>), two_axes(slots * a.Hk * p.splits), dim3(256), 0, st, a, slots);
    if (p.splits > 1) hipLaunchKernelGGL((k_attend_join<T>), two_axes(slots * a.Hk), dim3(256), 0, st, a, slots);
  } else {
    const long long slots = a.Tq * a.group / 128 + a.S;
    hipLaunchKernelGGL((k_attend<T, DP>), two_axes(slots * a.Hk), dim3(256), 0, st, a, slots);
  }
}

hipError_t launch_attention(const tdq_heads* Q, const tdq_heads* K, const tdq_heads* V, tdq_dtype dt, long long Tq,
                            long long Tk, int S, const int* cu_q, const int* cu_k, const int* len_k, int Hq, int Hk,
                            int D, float scale, bool causal, const tdq_heads* O, float* lse, void* workspace, hipStream_t st) {
  const AttendPlan p = attend_plan(Tq, Tk, S, Hq, Hk);
  AttendArgs a;
  a.Q = Q->data;
  a.K = K->data;
  a.V = V->data;
  a.O = O->data;
  a.lse = lse;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.len_k = len_k;
  a.q_token = Q->token;
  a.q_head = Q->head;
  a.k_token = K->token;
  a.k_head = K->head;
  a.v_token = V->token;
  a.v_head = V->head;
  a.o_token = O->token;
  a.o_head = O->head;
  a.Tq = Tq;
  a.Tk = Tk;
  a.S = S;
  a.Hq = Hq;
  a.Hk = Hk;
  a.group = Hq / Hk;
  a.D = D;
  a.causal = causal;
  const double c = fabs((double)scale) * 1.44269504088896340736;
  a.scale_log2 = c > 1e-30 ? (float)c : 1e-30f;
  a.lift = (dt == TDQ_F16 ? kLift<_Float16> : kLift<__bf16>) / a.scale_log2;
  a.flip = scale < 0.f ? 0x80008000u : 0u;
  a.splits = p.splits;
  a.part_ml = static_cast<float*>(workspace);
  a.part_o = p.splits > 1 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + part_ml_bytes(Tq, Hq, p.splits))
                          : nullptr;
#define TDQ_ATTEND(T)                                  \
  do {                                                 \
    if (D <= 32) launch_attend<T, 32>(a, p, st);       \
    else if (D <= 64) launch_attend<T, 64>(a, p, st);  \
    else if (D <= 128) launch_attend<T, 128>(a, p, st); \
    else launch_attend<T, 256>(a, p, st);              \
  } while (0)
  if (dt == TDQ_F16) TDQ_ATTEND(_Float16);
  else TDQ_ATTEND(__bf16);
#undef TDQ_ATTEND
  return hipGetLastError();
}

}  // namespace tdq
