// Linear in 8-bit floating point with one step for each block of 128.
//
//   codes   step = max(max |x|, 1e-8) / 448 over a block, q = e4m3(x / step): a block is 128
//           channels of one token (activations) or 128 outputs x 128 channels (weights)
//   linear  Y[m, n] = sum over blocks b of 128 channels of
//             x_step[m, b] * w_step[n / 128, b] * sum_{i in b} qx[m, i] qw[n, i]   (+ bias[n])
//
// 448 is the largest e4m3 value, so x / step never leaves the type's range.
#include "tdq_half.hpp"

namespace tdq {

constexpr int G8 = 128;                // channels of a block
constexpr float kE4m3Max = 448.0f;
constexpr float kStepFloor = 1e-8f;

// ---------------------------------------------------------------------------
// codes
// ---------------------------------------------------------------------------
// Step of a block from the largest magnitude's bits.  Compared as bits, a NaN is the largest of
// all: a block that holds one gets a NaN step, and one that holds an infinity an infinite step
// and NaN codes, so that the outputs of its row are not finite.
struct Step {
  float step, rcp;
  __device__ explicit Step(u32 max_bits) {
    const u32 floor_bits = __float_as_uint(kStepFloor);
    step = __uint_as_float(max_bits > floor_bits ? max_bits : floor_bits) / kE4m3Max;
    rcp = 1.0f / step;
  }
  // x / step correctly rounded: one correction of x * rcp by the exact remainder, rcp being the
  // correctly rounded reciprocal (3 instructions instead of the division's 10).  With these signs
  // a zero keeps its own.
  __device__ __forceinline__ float over(float x) const {
    const float q = x * rcp;
    return fmaf(-fmaf(q, step, -x), rcp, q);
  }
  __device__ __forceinline__ u32x2 codes(const float (&x)[8]) const {
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int v = 0;
      v = __builtin_amdgcn_cvt_pk_fp8_f32(over(x[4 * i]), over(x[4 * i + 1]), v, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(over(x[4 * i + 2]), over(x[4 * i + 3]), v, true);
      w[i] = (u32)v;
    }
    return w;
  }
};

// Eight elements from column c of a row of K on, zeros past its end.
template <typename T>
__device__ __forceinline__ void load_eight(const T* row, int c, int K, float (&x)[8]) {
  if (c + 8 <= K) {
    load_floats<T, 8>(row + c, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c + i < K ? (float)row[c + i] : 0.f;
  }
}

__device__ __forceinline__ u32 max_bits(const float (&x)[8]) {
  u32 m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const u32 b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = m > b ? m : b;
  }
  return m;
}

// Division by a launch constant of numbers below 2^31: n / d = (n * mul) >> 32 >> shift.
struct Divider {
  u32 mul, shift;
};
static Divider make_divider(u32 d) {
  Divider v;
  int s = 0;
  while ((1ull << s) < d) ++s;
  v.mul = s == 0 ? 0u : (u32)((((unsigned long long)1 << (31 + s)) + d - 1) / d);
  v.shift = s == 0 ? 0u : (u32)(s - 1);
  return v;
}
__device__ __forceinline__ u32 divide(u32 n, const Divider& d) {
  return d.mul == 0 ? n : __umulhi(n, d.mul) >> d.shift;
}

// One block of 128 channels of one row by 16 lanes, 8 channels each: a sweep bound by memory
// (131072 x 4096 bfloat16 in 281 us, 5.8 TB/s).
constexpr int kRowBlocks = 4;          // blocks per 16 lanes, all loaded before the first is used
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_f8_rows(const T* __restrict__ X, long long ld_x, u32 blocks, int K,
                                                          Divider per_row, int KB, uint8_t* __restrict__ Q,
                                                          long long ld_q, float* __restrict__ step, long long ld_s) {
  const int sub = threadIdx.x & 15;
  const u32 first = (blockIdx.x + blockIdx.y * gridDim.x) * (16u * kRowBlocks) + (threadIdx.x >> 4);
  float x[kRowBlocks][8];
  u32 row[kRowBlocks];
  int c[kRowBlocks];
#pragma unroll
  for (int u = 0; u < kRowBlocks; ++u) {
    const u32 b = first + 16u * u;
    if (b < blocks) {
      row[u] = divide(b, per_row);
      c[u] = (int)(b - row[u] * KB) * G8 + 8 * sub;
      load_eight(X + row[u] * ld_x, c[u], K, x[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < kRowBlocks; ++u) {
    if (first + 16u * u >= blocks) break;              // (the same in all 16 lanes)
    u32 m = max_bits(x[u]);
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) {
      const u32 o = __shfl_xor(m, d, 16);
      m = m > o ? m : o;
    }
    const Step s(m);
    if (c[u] < ((K + 15) & ~15)) *reinterpret_cast<u32x2*>(Q + row[u] * ld_q + c[u]) = s.codes(x[u]);
    if (sub == 0) step[row[u] * ld_s + c[u] / G8] = s.step;
  }
}

// A 128 x 128 tile of a weight by 256 threads, 64 elements each, held between the two looks: read
// once (4096 x 1024 binary32 in 7 us, most of it the launch).
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_f8_tiles(const T* __restrict__ W, long long ld_in, int N, int K,
                                                           uint8_t* __restrict__ Q, long long ld_q,
                                                           float* __restrict__ step, long long ld_s) {
  __shared__ u32 part[4];
  const int kb = blockIdx.x, nb = blockIdx.y;
  const int c = kb * G8 + 8 * (threadIdx.x & 15), r0 = nb * G8 + (threadIdx.x >> 4);
  float x[8][8];
  u32 m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < N) {
      load_eight(W + r * ld_in, c, K, x[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const u32 b = max_bits(x[i]);
    m = m > b ? m : b;
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const u32 o = __shfl_xor(m, d, 64);
    m = m > o ? m : o;
  }
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) m = m > part[i] ? m : part[i];
  const Step s(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < N && c < ((K + 15) & ~15)) *reinterpret_cast<u32x2*>(Q + r * ld_q + c) = s.codes(x[i]);
  }
  if (threadIdx.x == 0) step[nb * ld_s + kb] = s.step;
}

hipError_t launch_quantize_f8_rows(const void* X, tdq_dtype dt, long long M, int K, long long ld_x, uint8_t* Q,
                                   long long ld_q, float* step, long long ld_s, hipStream_t st) {
  const int KB = (K + G8 - 1) / G8;
  const u32 blocks = (u32)(M * KB);                    // below 2^31, checked by the caller
  const dim3 grid = two_axes(((long long)blocks + 16 * kRowBlocks - 1) / (16 * kRowBlocks));
  const Divider per_row = make_divider((u32)KB);
#define TDQ_ROWS(T)                                                                                              \
  hipLaunchKernelGGL((k_quantize_f8_rows<T>), grid, dim3(256), 0, st, static_cast<const T*>(X), ld_x, blocks, \
                     K, per_row, KB, Q, ld_q, step, ld_s)
  if (dt == TDQ_F16) TDQ_ROWS(_Float16);
  else if (dt == TDQ_BF16) TDQ_ROWS(__bf16);
  else TDQ_ROWS(float);
#undef TDQ_ROWS
  return hipGetLastError();
}

hipError_t launch_quantize_f8_tiles(const void* W, tdq_dtype dt, int N, int K, long long ld_in, uint8_t* Q,
                                    long long ld_q, float* step, long long ld_s, hipStream_t st) {
  const dim3 grid((K + G8 - 1) / G8, (N + G8 - 1) / G8);
#define TDQ_TILES(T)                                                                                               \
  hipLaunchKernelGGL((k_quantize_f8_tiles<T>), grid, dim3(256), 0, st, static_cast<const T*>(W), ld_in, N, K, Q, \
                     ld_q, step, ld_s)
  if (dt == TDQ_F16) TDQ_TILES(_Float16);
  else if (dt == TDQ_BF16) TDQ_TILES(__bf16);
  else TDQ_TILES(float);
#undef TDQ_TILES
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// linear
// ---------------------------------------------------------------------------
// Bytes [at, at + 4) of a row: those at K and beyond become code 0.
__device__ __forceinline__ void mask_codes(u32& w, int at, int K) {
  const int keep = K - at;
  if (keep < 4) w = keep <= 0 ? 0u : w & ((1u << (8 * keep)) - 1u);
}

// Eight codes as binary16 (exact: e4m3's values are binary16 values).
__device__ __forceinline__ h16x8 codes_to_half(u32 lo, u32 hi) {
  const h16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
  const h16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const h16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
  const h16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return h16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The sum of one block's products of a 16 x 16 piece of Y.
//   fine = false: one 16x16x128 matrix instruction on the codes.  It adds the products of a few
//     neighbouring channels with about 16 bits below the largest of them: measured, 1.3e-5 to
//     2.2e-5 of the result's norm, a tenth or less of what rounding a binary16 result costs.
//   fine = true (binary32 results): the codes as binary16, four 16x16x32 instructions of half
//     the rate, whose sums are as exact as binary32 (1e-8).
template <bool FINE>
__device__ __forceinline__ f32x4 block_sum(const i32x8& w, const i32x8& x) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  if constexpr (!FINE) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
  } else {
    f32x4 d = zero;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      d = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half(w[2 * g], w[2 * g + 1]),
                                                 codes_to_half(x[2 * g], x[2 * g + 1]), d, 0, 0, 0);
    return d;
  }
}

// The same of a 32 x 32 piece: two 32x32x64 instructions, or eight 32x32x16 on binary16.  (Half as
// many operand bytes per product as the 16 x 16 instruction.)
struct Frag {
  i32x8 k[2];                          // 64 channels each, in the order of the 16-byte pieces h, 2 + h | 4 + h, 6 + h
};
template <bool FINE>
__device__ __forceinline__ f32x16 block_sum(const Frag& w, const Frag& x) {
  f32x16 d;
#pragma unroll
  for (int i = 0; i < 16; ++i) d[i] = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (!FINE) {
      d = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w.k[k], x.k[k], d, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g)
        d = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_half(w.k[k][2 * g], w.k[k][2 * g + 1]),
                                                   codes_to_half(x.k[k][2 * g], x.k[k][2 * g + 1]), d, 0, 0, 0);
    }
  }
  return d;
}

// A run of 16 bytes of results, of which the first `left` elements are inside the row.  Past the
// caches: nothing reads Y here again, and it would push the operands out of the L2.
template <typename OUT>
__device__ __forceinline__ void store_run(OUT* p, u32x4 v, int left) {
  constexpr int V = 16 / sizeof(OUT);
  if (left >= V) {
    __builtin_nontemporal_store((u32x4_any)v, reinterpret_cast<u32x4_any*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i < left) {
        if constexpr (sizeof(OUT) == 4) p[i] = __uint_as_float(v[i]);
        else p[i] = __builtin_bit_cast(OUT, (u16)(v[i / 2] >> (16 * (i & 1))));
      }
    }
  }
}

// Workgroup tile (32 TM WM) x (32 TN WN) of Y, a wavefront's part (32 TM) x (32 TN).  The weight
// is the row operand of the matrix instruction: a lane's results are outputs of ONE token, so a
// block's rescale needs one step product per 32 tokens and lane.
// LDS: rows of 128 codes (one block), the 16-byte piece p of row r at position p ^ (r / 2 % 8):
// the 16 rows that a fragment read takes at a time fall on 16 different groups of banks.
// At 8192^3 (483 us, 2.3 PFLOP/s) the matrix units work 58 % of the cycles, at 1.9 GHz under this
// load: a block's start costs all wavefronts at once.  131072 x 1024 x 4096 (655 us, 1.7 PFLOP/s) has
// as many products and 42 %: of the 20 us of a tile 6 are its start and end, which nothing covers, and
// the stage that is copied behind the last block and not used.
template <typename OUT, bool FINE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_linear_f8(
    const uint8_t* __restrict__ Qx, long long ld_q, const float* __restrict__ xs, long long ld_xs, int M, int K, int N,
    const uint8_t* __restrict__ Qw, long long ld_w, const float* __restrict__ ws, long long ld_ws,
    const float* __restrict__ bias, OUT* __restrict__ Y, long long ld_y, int m_tiles, int n_tiles) {
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, WAVES = WM * WN;
  constexpr int CHUNKS = (BM + BN) / 8;                // of 8 rows, one copy instruction each
  static_assert(CHUNKS % WAVES == 0 && BM % 8 == 0 && (BM <= 64 || BM % 64 == 0), "copies of a stage");
  __shared__ __attribute__((aligned(1024))) uint8_t stage[2][(BM + BN) * G8];
  __shared__ float steps[2][BM < 64 ? 64 : BM];

  // Workgroups are dealt to the 8 XCDs in turn, each with its own L2.  Every XCD gets a run of the
  // tiles in an order that goes through bands of GM rows of tiles column by column, so that the 32
  // at work at a time share 8 + 4 pieces of the operands (all in one row: 1 + 32).
  constexpr int GM = 8;
  const long long bid = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const long long tiles = (long long)m_tiles * n_tiles, run = (tiles + 7) / 8;
  const long long order = (bid & 7) * run + (bid >> 3);
  if ((bid >> 3) >= run || order >= tiles) return;
  const int band = (int)(order / ((long long)GM * n_tiles));
  const int rest = (int)(order - (long long)band * GM * n_tiles);
  const int high = m_tiles - band * GM < GM ? m_tiles - band * GM : GM;
  const int m0 = (band * GM + rest % high) * BM, n0 = rest / high * BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int KB = (K + G8 - 1) / G8, last_piece = ((K + 15) / 16 - 1) * 16;
  const uint8_t* xb = Qx + m0 * ld_q;
  const uint8_t* wb = Qw + n0 * ld_w;
  const u32 lds0 = lds_address(&stage[0][0]), steps0 = lds_address(&steps[0][0]);

  // offsets of the rows that this lane copies, and of its piece within a block
  u32 row_off[CHUNKS / WAVES];
  const int sub = lane >> 3;
#pragma unroll
  for (int i = 0; i < CHUNKS / WAVES; ++i) {
    const int c = wave + i * WAVES, r = c * 8 + sub;
    if (r < BM) {
      const int m = r < M - m0 ? r : M - 1 - m0;
      row_off[i] = (u32)(m * ld_q);
    } else {
      const int n = r - BM < N - n0 ? r - BM : N - 1 - n0;
      row_off[i] = (u32)(n * ld_w);
    }
  }
  const int sm = (wave * 64 + lane) < M - m0 ? wave * 64 + lane : M - 1 - m0;
  const u32 step_off = (u32)(sm * ld_xs * 4);
  // One of the TM parts of stage kb.
  auto copy_part = [&](int kb, int part) {
    constexpr int ALL = CHUNKS / WAVES, EACH = (ALL + TM - 1) / TM;
    const u32 base = lds0 + (u32)(kb & 1) * ((BM + BN) * G8);
#pragma unroll
    for (int i = part * EACH; i < (part + 1) * EACH && i < ALL; ++i) {
      const int c = wave + i * WAVES;
      // (chunk rows 8 c ..: row r has its pieces turned by r / 2 % 8, r = 8 c + sub)
      int at = kb * G8 + 16 * ((lane & 7) ^ ((4 * c + (sub >> 1)) & 7));
      at = at < last_piece ? at : last_piece;
      copy_to_lds(c * 8 < BM ? xb : wb, row_off[i] + at, base + c * 1024);
    }
    if (part == 0 && wave * 64 < BM)
      copy_float_to_lds(xs + m0 * ld_xs + (kb < KB ? kb : KB - 1), step_off,
                        steps0 + (u32)((kb & 1) * (BM < 64 ? 64 : BM) + wave * 64) * 4);
  };

  f32x16 acc[TN][TM];
#pragma unroll
  for (int u = 0; u < TN; ++u)
#pragma unroll
    for (int t = 0; t < TM; ++t) acc[u][t] = f32x16{};

  // A fragment: row lane % 32, the 16-byte pieces 2 j + lane / 32.  Both operands name the channels
  // in this order, so it does not matter which.
  const int fr = lane & 31, fh = lane >> 5, turn = (fr >> 1) & 7;
  const int off = fr * G8 + 16 * (fh ^ turn);          // piece 2 j + fh: off ^ 32 j
  const float* wsp = ws + ((n0 + wn * 32 * TN) / G8) * ld_ws;
  if (n0 + wn * 32 * TN >= N) wsp = ws;                // (nothing of such a wavefront is stored)

#pragma unroll
  for (int t = 0; t < TM; ++t) copy_part(0, t);
  float w_next = wsp[0];
  for (int kb = 0; kb < KB; ++kb) {
    wait_copies();
    __syncthreads();
    const uint8_t* sx = &stage[kb & 1][wm * 32 * TM * G8];
    const uint8_t* sw = &stage[kb & 1][(BM + wn * 32 * TN) * G8];
    const float w_step = w_next;                       // (asked for a block ahead)
    w_next = wsp[kb + 1 < KB ? kb + 1 : kb];
    if ((kb + 1) * G8 > K) {                           // (the last block, cut: code 0 from K on)
      const int real = K - kb * G8;
      for (int i = threadIdx.x; i < (BM + BN) * 8; i += 64 * WAVES) {
        const int r = i >> 3, piece = (i & 7) ^ ((r >> 1) & 7), keep = real - 16 * piece;
        if (keep < 16) {
          u32* w = reinterpret_cast<u32*>(&stage[kb & 1][16 * i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) mask_codes(w[j], 4 * j, keep);
        }
      }
      __syncthreads();
    }
    auto fragment = [&](const uint8_t* p) {
      Frag f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(p + (off ^ (64 * k)));
        const u32x4 b = *reinterpret_cast<const u32x4*>(p + (off ^ (64 * k + 32)));
        f.k[k] = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
      }
      return f;
    };
    Frag fw[TN];
#pragma unroll
    for (int u = 0; u < TN; ++u) fw[u] = fragment(sw + u * 32 * G8);
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      const Frag fx = fragment(sx + t * 32 * G8);
      copy_part(kb + 1, t);
      const float s = steps[kb & 1][(wm * TM + t) * 32 + fr] * w_step;
#pragma unroll
      for (int u = 0; u < TN; ++u) {
        const f32x16 d = block_sum<FINE>(fw[u], fx);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[u][t][i] = fmaf(d[i], s, acc[u][t][i]);
      }
      // (keeps the compiler from reading all fragments at once, which spills)
      if (TM * TN > 4) __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Results: 32 rows at a time through a piece of LDS of the wavefront's own, so that a store
  // instruction writes whole runs of 64 TN (binary16) or 128 TN bytes of each row.
  wait_copies();                                       // (one stage past the last, never read)
  __syncthreads();
  constexpr int COLS = 32 * TN, V = 16 / sizeof(OUT), LANES = COLS / V;      // lanes that store a row's run
  static_assert(32 * (COLS + V) * sizeof(OUT) * WAVES <= sizeof(stage), "room for the results");
  OUT* out = reinterpret_cast<OUT*>(&stage[0][0]) + wave * 32 * (COLS + V);
  const int nw = n0 + wn * COLS;
  float b[TN][16];                                     // (read once, for all of the wavefront's tokens)
#pragma unroll
  for (int u = 0; u < TN; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int n = nw + 32 * u + 8 * (i / 4) + 4 * fh + i % 4;
      b[u][i] = bias && n < N ? bias[n] : 0.f;
    }
#pragma unroll
  for (int t = 0; t < TM; ++t) {
#pragma unroll
    for (int u = 0; u < TN; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = 32 * u + 8 * q + 4 * fh;
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = bias ? acc[u][t][4 * q + i] + b[u][4 * q + i] : acc[u][t][4 * q + i];
        store_floats<OUT, 4>(out + fr * (COLS + V) + c, y);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 32; i += 64 / LANES) {
      const int r = i + lane / LANES, c = lane % LANES * V;
      const int m = m0 + (wm * TM + t) * 32 + r, n = nw + c;
      const u32x4 v = *reinterpret_cast<const u32x4*>(out + r * (COLS + V) + c);
      if (m < M && n < N) store_run(Y + m * ld_y + n, v, N - n);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Few tokens: bound by reading the weight once.  A workgroup has 16 outputs and all tokens, its
// wavefronts share out the blocks of K: each reads its blocks of 16 x 128 codes straight to
// registers, a lane 32 bytes and four lanes a whole line, several blocks at a time, and the
// wavefronts' sums are joined in LDS.  One token, 4096 -> 4096: 5.8 us, by 64 x 64 tiles 14.
constexpr int kFewWaves = 8;
template <typename OUT, bool FINE, int TM>
__global__ __launch_bounds__(64 * kFewWaves) void k_linear_f8_few(
    const uint8_t* __restrict__ Qx, long long ld_q, const float* __restrict__ xs, long long ld_xs, int M, int K, int N,
    const uint8_t* __restrict__ Qw, long long ld_w, const float* __restrict__ ws, long long ld_ws,
    const float* __restrict__ bias, OUT* __restrict__ Y, long long ld_y) {
  constexpr int AHEAD = TM == 1 ? 4 : 2;               // blocks read at a time
  __shared__ f32x4 part[kFewWaves][TM][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fq = lane >> 4, n0 = blockIdx.x * 16;
  const int KB = (K + G8 - 1) / G8, last = ((K + 15) / 16 - 1) * 16;
  const uint8_t* wp = Qw + (long long)(n0 + fr < N ? n0 + fr : N - 1) * ld_w;
  const float* wsp = ws + (n0 / G8) * ld_ws;
  const uint8_t* xp[TM];
  const float* xsp[TM];
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int m = 16 * t + fr < M ? 16 * t + fr : M - 1;
    xp[t] = Qx + m * ld_q;
    xsp[t] = xs + m * ld_xs;
  }
  auto read = [&](const uint8_t* row, int kb) {
    const int at = kb * G8 + 32 * fq, a0 = at < last ? at : last, a1 = at + 16 < last ? at + 16 : last;
    const u32x4 a = *reinterpret_cast<const u32x4*>(row + a0), b = *reinterpret_cast<const u32x4*>(row + a1);
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
  };
  f32x4 acc[TM];
#pragma unroll
  for (int t = 0; t < TM; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = wave; k0 < KB; k0 += kFewWaves * AHEAD) {
    i32x8 fw[AHEAD], fx[AHEAD][TM];
    float s[AHEAD][TM];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int kb = k0 + kFewWaves * j;
      if (kb < KB) {                                   // (the same in every lane)
        fw[j] = read(wp, kb);
        const float w_step = wsp[kb];
#pragma unroll
        for (int t = 0; t < TM; ++t) {
          fx[j][t] = read(xp[t], kb);
          s[j][t] = xsp[t][kb] * w_step;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int kb = k0 + kFewWaves * j;
      if (kb >= KB) break;
      if ((kb + 1) * G8 > K) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u32 w = (u32)fw[j][i];
          mask_codes(w, kb * G8 + 32 * fq + 4 * i, K);
          fw[j][i] = (int)w;
#pragma unroll
          for (int t = 0; t < TM; ++t) {
            u32 x = (u32)fx[j][t][i];
            mask_codes(x, kb * G8 + 32 * fq + 4 * i, K);
            fx[j][t][i] = (int)x;
          }
        }
      }
#pragma unroll
      for (int t = 0; t < TM; ++t) {
        const f32x4 d = block_sum<FINE>(fw[j], fx[j][t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(d[i], s[j][t], acc[t][i]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < TM; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  // wavefront t adds the parts of tokens 16 t ..
  for (int t = wave; t < TM; t += kFewWaves) {
    f32x4 y = part[0][t][lane];
#pragma unroll
    for (int v = 1; v < kFewWaves; ++v) y += part[v][t][lane];
    const int m = 16 * t + fr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + 4 * fq + i;
      if (m < M && n < N) Y[m * ld_y + n] = (OUT)(bias ? y[i] + bias[n] : y[i]);
    }
  }
}

template <typename OUT, bool FINE, int TM, int TN, int WM, int WN>
static void launch_linear(const uint8_t* Qx, long long ld_q, const float* xs, long long ld_xs, int M, int K, int N,
                          const uint8_t* Qw, long long ld_w, const float* ws, long long ld_ws, const float* bias,
                          void* Y, long long ld_y, hipStream_t st) {
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN;
  const int m_tiles = (M + BM - 1) / BM, n_tiles = (N + BN - 1) / BN;
  const dim3 grid = two_axes(((long long)m_tiles * n_tiles + 7) / 8 * 8);
  hipLaunchKernelGGL((k_linear_f8<OUT, FINE, TM, TN, WM, WN>), grid, dim3(64 * WM * WN), 0, st, Qx, ld_q, xs, ld_xs, M,
                     K, N, Qw, ld_w, ws, ld_ws, bias, static_cast<OUT*>(Y), ld_y, m_tiles, n_tiles);
}

// The kernel for a shape: up to 32 tokens the one that reads the weight straight to registers, else
// the tile whose time is least, by what a block of K took (us), with one round of tiles and with
// many:
//   64 x 64    0.44 up to 256 tiles (128 x 4096 x 4096: 14.2), then 0.94 for each 1000; binary32 0.57, 1.4
//   128 x 256  1.15 for each 256 tiles; binary32 1.9
//   256 x 256  1.75 for each 256 tiles (8192 x 8192 x 8192: 472, 128 x 256 586, 64 x 64 951)
//   128 x 128  (binary32, whose operands as binary16 spill from a 256 x 256 tile) 1.17, 4.3 for each 1000
// No tile cuts K, so that few tiles over a long K leave most of the chip idle: 4096 x 4096 takes 9.7 us
// with 32 tokens and 13.8 with 33 (floor 2.7), 8192 -> 1024 25 us with 64, 4096 -> 512 14 us with 968.
enum { kFew16, kFew32, k64x64, k128x256, kLargest };
static int linear_way(long long M, long long N, bool fine) {
  if (M <= 32) return M <= 16 ? kFew16 : kFew32;
  auto tiles = [&](long long bm, long long bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  auto at_least = [](double most, double least) { return most > least ? most : least; };
  auto rounds = [](long long n) { return (double)((n + 255) / 256); };
  const double small = fine ? at_least(1.4e-3 * tiles(64, 64), 0.57) : at_least(0.94e-3 * tiles(64, 64), 0.44);
  const double middle = (fine ? 1.9 : 1.15) * rounds(tiles(128, 256));
  const double large = fine ? at_least(4.3e-3 * tiles(128, 128), 1.17) : 1.75 * rounds(tiles(256, 256));
  return small <= middle && small <= large ? k64x64 : middle <= large ? k128x256 : kLargest;
}

hipError_t launch_linear_f8(const uint8_t* Qx, long long ld_q, const float* xs, long long ld_xs, int M, int K, int N,
                            const uint8_t* Qw, long long ld_w, const float* ws, long long ld_ws, const float* bias,
                            void* Y, tdq_dtype y_dt, long long ld_y, hipStream_t st) {
  const int way = linear_way(M, N, y_dt == TDQ_F32);
#define TDQ_TILE(OUT, FINE, TM, TN, WM, WN) \
  launch_linear<OUT, FINE, TM, TN, WM, WN>(Qx, ld_q, xs, ld_xs, M, K, N, Qw, ld_w, ws, ld_ws, bias, Y, ld_y, st)
#define TDQ_FEW(OUT, FINE, TM)                                                                                      \
  hipLaunchKernelGGL((k_linear_f8_few<OUT, FINE, TM>), dim3((N + 15) / 16), dim3(64 * kFewWaves), 0, st, Qx, ld_q, \
                     xs, ld_xs, M, K, N, Qw, ld_w, ws, ld_ws, bias, static_cast<OUT*>(Y), ld_y)
#define TDQ_LINEAR(OUT, FINE)                                    \
  do {                                                           \
    if (way == kFew16) TDQ_FEW(OUT, FINE, 1);                    \
    else if (way == kFew32) TDQ_FEW(OUT, FINE, 2);               \
    else if (way == k64x64) TDQ_TILE(OUT, FINE, 1, 1, 2, 2);     \
    else if (way == k128x256) TDQ_TILE(OUT, FINE, 2, 2, 2, 4);   \
    else if constexpr (FINE) TDQ_TILE(OUT, FINE, 2, 2, 2, 2);    \
    else TDQ_TILE(OUT, FINE, 4, 2, 2, 4);                        \
  } while (0)
  if (y_dt == TDQ_F16) TDQ_LINEAR(_Float16, false);
  else if (y_dt == TDQ_BF16) TDQ_LINEAR(__bf16, false);
  else TDQ_LINEAR(float, true);
#undef TDQ_LINEAR
  return hipGetLastError();
}

}  // namespace tdq
