// Norm of query and key heads with the rotation by position, and softmax attention with grouped
// heads over packed sequences.
#include "tdq_half.hpp"

namespace tdq {

// ---------------------------------------------------------------------------
// norm and rotation
// ---------------------------------------------------------------------------
// y = x / sqrt(mean x^2 + eps) * w over a head's D elements, then pair p of the first R by the
// angle pos[axis of p] * freq[p]:  (a, b) -> (a cos - b sin, b cos + a sin).
// One pass: the rows are read and written once, bound by memory.  The angles of a token serve
// all its heads, so a workgroup takes a few whole tokens and leaves their cosines and sines in
// LDS.  An angle is reduced as a fraction of a turn in binary64: a binary32 product of a
// position of 100000 is off by up to 0.004 radians, more than bfloat16's rounding.
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
  const long long t0 = (long long)blockIdx.x * tokens;
  const int here = (int)(a.T - t0 < tokens ? a.T - t0 : tokens);
  for (int i = threadIdx.x; i < here * P; i += kRotateThreads) {
    const int t = i / P, p = i - t * P;
    int ax = a.axis ? a.axis[p] : 0;
    ax = ax < 0 ? 0 : ax < a.axes ? ax : a.axes - 1;
    const double turns = (double)a.pos[ax * a.ld_pos + t0 + t] * ((double)a.freq[p] * 0.15915494309189533577);
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    turn[t][2 * p] = c;
    turn[t][2 * p + 1] = s;
  }
  __syncthreads();
  const int sub = threadIdx.x & (L - 1), heads = a.heads[0] + a.heads[1];
  const int D = a.D, R = a.R;
  const bool mine = 8 * sub < D, turned = 8 * sub < R;
  // 8 elements of a lane: neighbours, or 4 of the first half of the turned ones and their partners
  const int e0 = PAIRS || !turned ? 8 * sub : 4 * sub, e1 = PAIRS || !turned ? e0 + 4 : P + 4 * sub;
  for (int i = threadIdx.x / L; i < here * heads; i += kRotateThreads / L) {
    const int t = i / heads, hh = i - t * heads, which = hh >= a.heads[0], h = which ? hh - a.heads[0] : hh;
    const T* src = static_cast<const T*>(a.in[which]) + (t0 + t) * a.in_token[which] + h * a.in_head[which];
    T* dst = static_cast<T*>(a.out[which]) + (t0 + t) * a.out_token[which] + h * a.out_head[which];
    const float* w = a.weight[which];
    float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
      load_floats<T, 4>(src + e0, x);
      load_floats<T, 4>(src + e1, y);
    }
    if (w) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum = fmaf(x[j], x[j], fmaf(y[j], y[j], sum));
#pragma unroll
      for (int d = L / 2; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, L);
      const float r = 1.0f / sqrtf(sum / (float)D + a.eps);
      if (mine) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = x[j] * r * w[e0 + j];
          y[j] = y[j] * r * w[e1 + j];
        }
      }
    }
    if (turned) {
      const float* cs = &turn[t][8 * sub];
      float z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = cs[j];
      if constexpr (PAIRS) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float p = x[2 * j], q = x[2 * j + 1], u = y[2 * j], v = y[2 * j + 1];
          x[2 * j] = fmaf(p, z[2 * j], -(q * z[2 * j + 1]));
          x[2 * j + 1] = fmaf(q, z[2 * j], p * z[2 * j + 1]);
          y[2 * j] = fmaf(u, z[4 + 2 * j], -(v * z[5 + 2 * j]));
          y[2 * j + 1] = fmaf(v, z[4 + 2 * j], u * z[5 + 2 * j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = x[j], q = y[j];
          x[j] = fmaf(p, z[2 * j], -(q * z[2 * j + 1]));
          y[j] = fmaf(q, z[2 * j], p * z[2 * j + 1]);
        }
      }
    }
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
  const unsigned grid = (unsigned)((T + tokens - 1) / tokens);
#define TDQ_ROTATE_LP(T_, L, PAIRS) \
  hipLaunchKernelGGL((k_norm_rotate<T_, L, PAIRS>), dim3(grid), dim3(kRotateThreads), 0, st, a, tokens)
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
// sum of the softmax (binary32):
//   S^T = K Q^T       keys x rows: a lane holds 16 of every 32 keys of ONE row, so that a row's
//                     maximum is 15 steps in the lane and one exchange of the two halves
//   P^T = 2^(c S^T - c m), rounded to the type of V as the matrix instruction's operand
//   O^T += V^T P^T    a lane's probabilities are its operand as they lie: the order of the keys
//                     within an instruction is free as long as V^T is read in the same order
// The sum of the probabilities is taken before their rounding.
struct AttendArgs {
  const void *Q, *K, *V;
  void* O;
  float* lse;
  const int *cu_q, *cu_k;
  long long q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  long long Tq, Tk;
  int S, Hq, Hk, group, D, causal;
  float scale_log2;                    // scale * log2(e)
};

// What keys and values past the end of a sequence, or past D, are copied from.
__device__ u32x4 kZeros[4];

template <typename T>
struct Mfma;
template <>
struct Mfma<_Float16> {
  typedef h16x8 frag;
  __device__ static __forceinline__ f32x16 mul(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(frag, a), __builtin_bit_cast(frag, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma<__bf16> {
  typedef b16x8 frag;
  __device__ static __forceinline__ f32x16 mul(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(frag, a), __builtin_bit_cast(frag, b), c, 0, 0, 0);
  }
};

__device__ __forceinline__ float other_half(float x) {   // the value of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
// Four elements down a column: 16 lanes give the addresses of 4 rows x 16 columns (a lane 4
// columns of row lane / 4), lane i gets column i.
__device__ __forceinline__ u32x2 read_column(u32 lds) {
  const s16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)lds);
  return __builtin_bit_cast(u32x2, r);
}

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

constexpr int kKeys = 64;              // keys of a tile

template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attend(AttendArgs a, long long slots) {
  constexpr int BM = 128, PIECES = DP / 8, ROW = DP * 2;     // 16-byte pieces and bytes of a row in LDS
  constexpr int ROWS_PER_COPY = 64 / PIECES, COPIES = kKeys / ROWS_PER_COPY / 4;   // per wavefront
  // Where piece c of row r lies, so that what is read at a time spreads over the banks: K by 16
  // rows of one piece, V by 4 rows of 64 bytes.
  auto place_k = [](int r) { return DP >= 128 ? r & 15 : DP == 64 ? (r >> 1) & 7 : (r >> 2) & 3; };
  auto place_v = [](int r) { return DP >= 128 ? 4 * (r & 3) : DP == 64 ? 4 * ((r >> 1) & 1) : 0; };
  __shared__ __attribute__((aligned(1024))) uint8_t sk[kKeys * ROW], sv[kKeys * ROW];

  const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  if (id >= slots * a.Hk) return;
  const int hk = (int)(id % a.Hk);
  const Slot slot = find_slot<BM>(a, slots - 1 - id / a.Hk);
  const int q0 = clamp_start(a.cu_q, slot.seq, a.Tq), nq = clamp_start(a.cu_q, slot.seq + 1, a.Tq) - q0;
  const int k0 = clamp_start(a.cu_k, slot.seq, a.Tk);
  int nk = clamp_start(a.cu_k, slot.seq + 1, a.Tk) - k0;
  nk = nk > 0 ? nk : 0;
  const long long rows = nq > 0 ? (long long)nq * a.group : 0;
  const long long r0 = (long long)slot.tile * BM;
  if (r0 >= rows) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, D = a.D;
  const int ahead = nk - nq;                           // a causal token t sees the keys up to t + ahead

  // this lane's row
  const long long row = r0 + wave * 32 + (lane & 31);
  const bool real = row < rows;
  const long long row_c = real ? row : rows - 1;
  const int token = (int)(row_c / a.group), head = hk * a.group + (int)(row_c - (long long)token * a.group);
  const int sees = a.causal ? (token + ahead + 1 < nk ? token + ahead + 1 : nk) : nk;   // keys that the row sees
  // and how many of the tile's keys the workgroup, and this wavefront, need
  long long last = r0 + BM - 1;
  if (last > rows - 1) last = rows - 1;
  int end = a.causal ? (int)(last / a.group) + ahead + 1 : nk;
  end = end < nk ? end : nk;
  end = __builtin_amdgcn_readfirstlane(end);

  u32x4 q[DP / 16];
  {
    const T* qp = static_cast<const T*>(a.Q) + (q0 + token) * a.q_token + head * a.q_head;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const int c = 16 * i + 8 * half;
      q[i] = u32x4{0, 0, 0, 0};
      if (c < D) q[i] = *reinterpret_cast<const u32x4*>(qp + c);
    }
  }
  f32x16 o[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m = -INFINITY, l = 0.f;                        // running maximum (of the row), sum (of this lane's keys)

  const T* kp = static_cast<const T*>(a.K) + k0 * a.k_token + hk * a.k_head;
  const T* vp = static_cast<const T*>(a.V) + k0 * a.v_token + hk * a.v_head;
  const u32 lk = lds_address(sk), lv = lds_address(sv);
  const int crow = lane / PIECES, cpos = lane % PIECES;
  for (int j0 = 0; j0 < end; j0 += kKeys) {
    __syncthreads();                                   // the last tile has been read
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const int c = wave * COPIES + i, r = c * ROWS_PER_COPY + crow;
      const int pk = cpos ^ place_k(r), pv = cpos ^ place_v(r);
      const T* sk_ = kp + (j0 + r) * a.k_token + 8 * pk;
      const T* sv_ = vp + (j0 + r) * a.v_token + 8 * pv;
      copy_to_lds(j0 + r < nk && 8 * pk < D ? (const void*)sk_ : (const void*)kZeros, lk + c * 1024);
      copy_to_lds(j0 + r < nk && 8 * pv < D ? (const void*)sv_ : (const void*)kZeros, lv + c * 1024);
    }
    wait_copies();
    __syncthreads();

    // scores: element i of s[n] is key 32 n + 8 (i / 4) + 4 half + i % 4
    f32x16 s[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int j = 0; j < 16; ++j) s[n][j] = 0.f;
      const int r = 32 * n + (lane & 31);
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        const u32x4 k = *reinterpret_cast<const u32x4*>(&sk[r * ROW + 16 * ((2 * i + half) ^ place_k(r))]);
        s[n] = Mfma<T>::mul(k, q[i], s[n]);
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int key = j0 + 32 * n + 8 * (j / 4) + 4 * half + j % 4;
        s[n][j] = key < sees ? s[n][j] * a.scale_log2 : -INFINITY;
        top = fmaxf(top, s[n][j]);
      }
    top = fmaxf(top, other_half(top));
    const float m_new = fmaxf(m, top);
    const float base = m_new == -INFINITY ? 0.f : m_new;       // (a row that has seen no key yet)
    const float keep = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    float sum = 0.f;
    u32 p[2][8];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[n][j] - base), p1 = __builtin_amdgcn_exp2f(s[n][j + 1] - base);
        sum += p0 + p1;
        p[n][j / 2] = two_rounded<T>(p0, p1);
      }
    l = fmaf(l, keep, sum);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] *= keep;
    // values: 16 keys at a time, a lane's 8 of them 4 half .. + 3 and 8 + 4 half .. + 3
    const int tr = lane & 15;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const u32x4 pb = {p[n / 2][4 * (n & 1)], p[n / 2][4 * (n & 1) + 1], p[n / 2][4 * (n & 1) + 2],
                        p[n / 2][4 * (n & 1) + 3]};
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) {
        const int c = 4 * i + 2 * ((lane >> 4) & 1) + ((tr & 3) >> 1);      // 16-byte piece of this lane's four columns
        const int ra = 16 * n + 4 * half + (tr >> 2), rb = ra + 8;
        const u32x2 va = read_column(lv + ra * ROW + 16 * (c ^ place_v(ra)) + 8 * (tr & 1));
        const u32x2 vb = read_column(lv + rb * ROW + 16 * (c ^ place_v(rb)) + 8 * (tr & 1));
        o[i] = Mfma<T>::mul(u32x4{va[0], va[1], vb[0], vb[1]}, pb, o[i]);
      }
    }
  }

  l += other_half(l);
  if (!real) return;
  const float inv = m == -INFINITY ? 0.f : 1.0f / l;   // a row that sees no key: zeros, and -inf
  T* op = static_cast<T*>(a.O) + (q0 + token) * a.o_token + head * a.o_head;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      const int c = 32 * i + 2 * j + 4 * half;
      if (c < D) {
        const float y[4] = {o[i][j] * inv, o[i][j + 1] * inv, o[i][j + 2] * inv, o[i][j + 3] * inv};
        store_floats<T, 4>(op + c, y);
      }
    }
  if (a.lse && half == 0)
    a.lse[(q0 + (long long)token) * a.Hq + head] =
        m == -INFINITY ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

template <typename T, int DP>
static void launch_attend(const AttendArgs& a, hipStream_t st) {
  const long long slots = a.Tq * a.group / 128 + a.S;
  const long long total = slots * a.Hk, axis = 1 << 22;
  const dim3 grid(total < axis ? (unsigned)total : (unsigned)axis, (unsigned)((total + axis - 1) / axis));
  hipLaunchKernelGGL((k_attend<T, DP>), grid, dim3(256), 0, st, a, slots);
}

size_t attention_workspace(long long, long long, int, int, int, int) { return 0; }

hipError_t launch_attention(const tdq_heads* Q, const tdq_heads* K, const tdq_heads* V, tdq_dtype dt, long long Tq,
                            long long Tk, int S, const int* cu_q, const int* cu_k, int Hq, int Hk, int D, float scale,
                            bool causal, const tdq_heads* O, float* lse, void*, hipStream_t st) {
  AttendArgs a;
  a.Q = Q->data;
  a.K = K->data;
  a.V = V->data;
  a.O = O->data;
  a.lse = lse;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
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
  a.scale_log2 = (float)((double)scale * 1.44269504088896340736);
#define TDQ_ATTEND(T)                                  \
  do {                                                 \
    if (D <= 32) launch_attend<T, 32>(a, st);          \
    else if (D <= 64) launch_attend<T, 64>(a, st);     \
    else if (D <= 128) launch_attend<T, 128>(a, st);   \
    else launch_attend<T, 256>(a, st);                 \
  } while (0)
  if (dt == TDQ_F16) TDQ_ATTEND(_Float16);
  else TDQ_ATTEND(__bf16);
#undef TDQ_ATTEND
  return hipGetLastError();
}

}  // namespace tdq
