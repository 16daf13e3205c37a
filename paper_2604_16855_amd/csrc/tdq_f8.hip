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

// One block of 128 channels of one row by 16 lanes, 8 channels each; a memory-bound sweep.
constexpr int kRowBlocks = 4;          // blocks per 16 lanes, all loaded before the first is used
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_f8_rows(const T* __restrict__ X, long long ld_x, u32 blocks, int K,
                                                          Divider per_row, int KB, uint8_t* __restrict__ Q,
                                                          long long ld_q, float* __restrict__ step, long long ld_s) {
  const int sub = threadIdx.x & 15;
  const u32 first = blockIdx.x * (16u * kRowBlocks) + (threadIdx.x >> 4);
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

// A 128 x 128 tile of a weight by 256 threads, 64 elements each, held between the two looks.
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
  const u32 grid = (blocks + 16 * kRowBlocks - 1) / (16 * kRowBlocks);
  const Divider per_row = make_divider((u32)KB);
#define TDQ_ROWS(T)                                                                                              \
  hipLaunchKernelGGL((k_quantize_f8_rows<T>), dim3(grid), dim3(256), 0, st, static_cast<const T*>(X), ld_x, blocks, \
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
// Bytes [at, at + 8) of a row: those at K and beyond become code 0.
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

// Workgroup tile (16 TM WM) x (16 TN WN) of Y, a wavefront's part (16 TM) x (16 TN).  The weight
// is the row operand of the matrix instruction: a lane's four results are four outputs of ONE
// token, so a block's rescale needs one step product per 16 tokens and lane.
// LDS: rows of 128 codes (one block), the 16-byte piece p of row r at position p ^ (r / 2 % 8):
// the 16 rows that a fragment read takes at a time fall on 16 different groups of banks.
template <typename OUT, bool FINE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_linear_f8(
    const uint8_t* __restrict__ Qx, long long ld_q, const float* __restrict__ xs, long long ld_xs, int M, int K, int N,
    const uint8_t* __restrict__ Qw, long long ld_w, const float* __restrict__ ws, long long ld_ws,
    const float* __restrict__ bias, OUT* __restrict__ Y, long long ld_y, int m_tiles, int n_tiles) {
  constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN, WAVES = WM * WN;
  constexpr int CHUNKS = (BM + BN) / 8;                // of 8 rows, one copy instruction each
  static_assert(CHUNKS % WAVES == 0 && BM % 8 == 0 && (BM <= 64 || BM % 64 == 0), "copies of a stage");
  __shared__ __attribute__((aligned(1024))) uint8_t stage[2][(BM + BN) * G8];
  __shared__ float steps[2][BM < 64 ? 64 : BM];

  const long long bid = blockIdx.x + (long long)blockIdx.y * gridDim.x;
  const int xcd = (int)(bid & 7);
  const long long idx = bid >> 3;
  const long long m_tile = (idx / n_tiles) * 8 + xcd;
  if (m_tile >= m_tiles) return;
  const int m0 = (int)m_tile * BM, n0 = (int)(idx % n_tiles) * BN;
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
  auto copy_stage = [&](int kb) {
    const u32 base = lds0 + (u32)(kb & 1) * ((BM + BN) * G8);
#pragma unroll
    for (int i = 0; i < CHUNKS / WAVES; ++i) {
      const int c = wave + i * WAVES;
      // (chunk rows 8 c ..: row r has its pieces turned by r / 2 % 8, r = 8 c + sub)
      int piece = 16 * ((lane & 7) ^ ((4 * c + (sub >> 1)) & 7));
      if (kb * G8 + piece > last_piece) piece = last_piece - kb * G8;
      copy_to_lds((c * 8 < BM ? xb : wb) + kb * G8, row_off[i] + piece, base + c * 1024);
    }
    if (wave * 64 < BM) copy_float_to_lds(xs + m0 * ld_xs + kb, step_off, steps0 + (u32)((kb & 1) * (BM < 64 ? 64 : BM) + wave * 64) * 4);
  };

  f32x4 acc[TN][TM];
#pragma unroll
  for (int u = 0; u < TN; ++u)
#pragma unroll
    for (int t = 0; t < TM; ++t) acc[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // a fragment: row lane % 16, channels 32 (lane / 16) .. + 32, two pieces
  const int fr = lane & 15, fq = lane >> 4;
  const int turn = (fr >> 1) & 7;
  const int off0 = fr * G8 + 16 * ((2 * fq) ^ turn), off1 = fr * G8 + 16 * ((2 * fq + 1) ^ turn);
  const float* wsp = ws + ((n0 + wn * 16 * TN) / G8) * ld_ws;
  if (n0 + wn * 16 * TN >= N) wsp = ws;                // (nothing of such a wavefront is stored)

  copy_stage(0);
  for (int kb = 0; kb < KB; ++kb) {
    wait_copies();
    __syncthreads();
    if (kb + 1 < KB) copy_stage(kb + 1);
    const uint8_t* sx = &stage[kb & 1][wm * 16 * TM * G8];
    const uint8_t* sw = &stage[kb & 1][(BM + wn * 16 * TN) * G8];
    const float w_step = wsp[kb];
    const int left = K - kb * G8 - 32 * fq;            // codes of this lane's fragments that are real
    auto fragment = [&](const uint8_t* p) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(p + off0), b = *reinterpret_cast<const u32x4*>(p + off1);
      i32x8 f = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
      if ((kb + 1) * G8 > K) {                         // (the same in every lane)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u32 w = (u32)f[i];
          mask_codes(w, 4 * i, left);
          f[i] = (int)w;
        }
      }
      return f;
    };
    i32x8 fw[TN];
#pragma unroll
    for (int u = 0; u < TN; ++u) fw[u] = fragment(sw + u * 16 * G8);
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      const i32x8 fx = fragment(sx + t * 16 * G8);
      const float s = steps[kb & 1][wm * 16 * TM + t * 16 + fr] * w_step;
#pragma unroll
      for (int u = 0; u < TN; ++u) {
        const f32x4 d = block_sum<FINE>(fw[u], fx);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[u][t][i] = fmaf(d[i], s, acc[u][t][i]);
      }
    }
  }

#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int m = m0 + wm * 16 * TM + t * 16 + fr;
#pragma unroll
    for (int u = 0; u < TN; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + (wn * TN + u) * 16 + 4 * fq + i;
        if (m < M && n < N) {
          float y = acc[u][t][i];
          if (bias) y = y + bias[n];
          Y[m * ld_y + n] = (OUT)y;
        }
      }
    }
  }
}

template <typename OUT, bool FINE, int TM, int TN, int WM, int WN>
static void launch_linear(const uint8_t* Qx, long long ld_q, const float* xs, long long ld_xs, int M, int K, int N,
                          const uint8_t* Qw, long long ld_w, const float* ws, long long ld_ws, const float* bias,
                          void* Y, long long ld_y, hipStream_t st) {
  constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN;
  const int m_tiles = (M + BM - 1) / BM, n_tiles = (N + BN - 1) / BN;
  // an axis of a grid holds fewer than 2^32 threads: two axes (workgroups past the last tile return)
  const long long tiles = (long long)((m_tiles + 7) / 8) * 8 * n_tiles, axis = 1 << 22;
  const dim3 grid(tiles < axis ? (unsigned)tiles : (unsigned)axis, (unsigned)((tiles + axis - 1) / axis));
  hipLaunchKernelGGL((k_linear_f8<OUT, FINE, TM, TN, WM, WN>), grid, dim3(64 * WM * WN), 0, st, Qx, ld_q, xs, ld_xs, M,
                     K, N, Qw, ld_w, ws, ld_ws, bias, static_cast<OUT*>(Y), ld_y, m_tiles, n_tiles);
}

hipError_t launch_linear_f8(const uint8_t* Qx, long long ld_q, const float* xs, long long ld_xs, int M, int K, int N,
                            const uint8_t* Qw, long long ld_w, const float* ws, long long ld_ws, const float* bias,
                            void* Y, tdq_dtype y_dt, long long ld_y, hipStream_t st) {
#define TDQ_LINEAR(OUT, FINE) \
  launch_linear<OUT, FINE, 2, 2, 2, 2>(Qx, ld_q, xs, ld_xs, M, K, N, Qw, ld_w, ws, ld_ws, bias, Y, ld_y, st)
  if (y_dt == TDQ_F16) TDQ_LINEAR(_Float16, false);
  else if (y_dt == TDQ_BF16) TDQ_LINEAR(__bf16, false);
  else TDQ_LINEAR(float, true);
#undef TDQ_LINEAR
  return hipGetLastError();
}

}  // namespace tdq
