// A wavefront's share of softmax attention: 32 rows of queries against tiles of keys and values in
// LDS, with the running maximum and sum of the softmax.  See tdq_attention.hip for the formulas.
#pragma once

#include <math.h>

#include "tdq_half.hpp"

namespace tdq {

// What keys and values past the end of a sequence, or past D, are copied from.
static __device__ u32x4 kZeros[4];

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
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(frag, a), __builtin_bit_cast(frag, b), c, 0, 0,
                                                   0);
  }
};

__device__ __forceinline__ float other_half(float x) {   // the value of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ __forceinline__ float max_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Whether a row with maximum m and sum l has no key, or none with a score above -inf.  The maximum
// alone does not say: it passes over NaN, which the sum does not.
__device__ __forceinline__ bool no_weight(float m, float l) { return m == -INFINITY && l == 0.f; }
// Octaves that the reference m is set below the largest score.
template <typename T>
constexpr int kLift = __is_same(T, _Float16) ? 7 : 0;
// Log of the sum of exp(scale * score).
__device__ __forceinline__ float log_sum(float m, float l, float scale_log2) {
  return no_weight(m, l) ? -INFINITY : fmaf(m, scale_log2, __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
// Four elements down a column: 16 lanes give the addresses of 4 rows x 16 columns (a lane 4
// columns of row lane / 4), lane i gets column i.
__device__ __forceinline__ u32x2 read_column(u32 lds) {
  const s16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)lds);
  return __builtin_bit_cast(u32x2, r);
}
__device__ __forceinline__ u32x4 read_lds16(u32 lds) {
  return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)lds;
}

// Where the 16-byte piece c of row r lies in a row of LDS (c ^ place), so that what an
// instruction reads at a time spreads over the banks: K by 16 rows of one piece, V by 4 rows of
// 64 bytes.
template <int DP>
__device__ __forceinline__ int place_k(int r) {
  return DP >= 128 ? r & 15 : DP == 64 ? (r >> 1) & 7 : (r >> 2) & 3;
}
template <int DP>
__device__ __forceinline__ int place_v(int r) {
  return DP >= 128 ? 4 * (r & 3) : DP == 64 ? 4 * ((r >> 1) & 1) : 0;
}

// The same for V read by Rows16: by 8 rows of 32 bytes.
template <int DP>
__device__ __forceinline__ int place_v16(int r) {
  return place_v<DP>(r) ^ (2 * ((r >> 2) & 1));
}

// A wavefront's 32 rows: their queries, and the softmax and output so far.  Rows of LDS have DP
// elements, a power of two, of which DC (a multiple of 32) are worked on.
template <typename T, int DP, int DC = DP>
struct Rows {
  u32x4 q[DC / 16];                    // operand columns: row lane % 32, elements 16 i + 8 (lane / 32) ..
  // element j of o[i]: row lane % 32, output 32 i + 8 (j / 4) + 4 (lane / 32) + j % 4
  f32x16 o[DC / 32];
  float m, l;                          // reference of the exponents (of the row), sum (of this lane's keys)

  // TOGETHER: all on their way at once, from where there are zeros past D; else each under a condition.  us so
  // and so: 4 prompts' parts in pages 282 and 319 (registers), windows 25.9 and 26.6; packed single tokens,
  // whose first keys are on their way by then, 232 and 229.
  template <bool TOGETHER = true>
  __device__ __forceinline__ void start(const T* qp, int D, u32 flip) {
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) {
      const int c = 16 * i + 8 * half;
      if (TOGETHER) {
        q[i] = *(c < D ? reinterpret_cast<const u32x4*>(qp + c) : reinterpret_cast<const u32x4*>(kZeros)) ^ flip;
      } else {
        q[i] = u32x4{0, 0, 0, 0};
        if (c < D) q[i] = *reinterpret_cast<const u32x4*>(qp + c) ^ flip;
      }
    }
#pragma unroll
    for (int i = 0; i < DC / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }

  // LDS addresses that this lane reads of a tile, of K's 16 elements i and of V's 32 outputs i; the
  // rows of a tile from 32 n on are at the same places 32 n rows further.
  u32 ka[DC / 16], va[DC / 32];
  __device__ __forceinline__ void addresses(u32 lk, u32 lv) {
    const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5, tr = lane & 15;
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) ka[i] = lk + row * (2 * DP) + 16 * ((2 * i + half) ^ place_k<DP>(row));
    const int key = 4 * half + (tr >> 2);              // (place_v is the same every four rows)
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) {
      const int c = 4 * i + 2 * ((lane >> 4) & 1) + ((tr & 3) >> 1);
      va[i] = lv + key * (2 * DP) + 16 * (c ^ place_v<DP>(key)) + 8 * (tr & 1);
    }
  }
  __device__ __forceinline__ void move(int by) {
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) ka[i] += by;
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) va[i] += by;
  }

  // Products of 32 keys from row r (a multiple of 32) of a tile on: element j is key
  // 8 (j / 4) + 4 (lane / 32) + j % 4.
  __device__ __forceinline__ f32x16 scores(int r) const {
    f32x16 s;
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) s = Mfma<T>::mul(read_lds16(ka[i] + r * (2 * DP)), q[i], s);
    return s;
  }

  // Scores -> probabilities, of N times 32 keys; `seen(k)`: whether the row sees key k of them (asked
  // only where `masked`).  lift: kLift octaves as a score.  The probabilities are rounded to the type of V, as the
  // matrix instructions take them, by half a step each; their sum is of the unrounded ones, in binary32.  With O's
  // own rounding outputs of bfloat16 lay 0.0017 to 0.0019 from 64 bits, relative to their norm, where ones by binary32
  // probabilities lay 0.0016 to 0.0017.
  template <int N, typename F>
  __device__ __forceinline__ void softmax(f32x16 (&s)[N], u32 (&p)[N][8], float c, float lift, bool masked, F seen) {
    const int half = (threadIdx.x >> 5) & 1;
    if (masked) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          s[n][j] = seen(32 * n + 8 * (j / 4) + 4 * half + j % 4) ? s[n][j] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, s[n][j]);
    top = max_of_halves(top);
    if (__ballot((top - m) * c > 8.0f + kLift<T> || (m == -INFINITY && top > m))) {
      const float m_new = fmaxf(m, kLift<T> == 0 ? top : top - lift);
      // (rows that have seen no key yet keep their zeros)
      const float keep = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - m_new) * c);
      m = m_new;
      l *= keep;
#pragma unroll
      for (int i = 0; i < DC / 32; ++i) {
        // In place: from an ordinary product the compiler makes a copy of all of O in every pass, 64
        // moves.  It does not see what these instructions read and write, so the wait states that it
        // would put between matrix instructions and them are here, tied to the values: 20 before the
        // first, as many as the longest matrix instruction needs, and two behind the last.
        asm volatile("s_nop 15\n\ts_nop 3" : "+v"(o[i]));
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          float e = o[i][j];
          asm volatile("v_mul_f32 %0, %1, %0" : "+v"(e) : "v"(keep));
          o[i][j] = e;
        }
        asm volatile("s_nop 1" : "+v"(o[i]));
      }
    }
    const float base = m == -INFINITY ? 0.f : -m * c;
    float sum = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[n][j], c, base));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[n][j + 1], c, base));
        sum += p0 + p1;
        p[n][j / 2] = two_rounded<T>(p0, p1);
      }
    l += sum;
  }

  // O^T += V^T P^T for 32 keys from row r (a multiple of 32) of a tile on: an operand has 16 keys,
  // a lane's 8 of them 4 half .. + 3 and 8 + 4 half .. + 3, as its probabilities lie.
  __device__ __forceinline__ void values(int r, const u32 (&p)[8]) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const u32x4 pb = {p[4 * n], p[4 * n + 1], p[4 * n + 2], p[4 * n + 3]};
#pragma unroll
      for (int i = 0; i < DC / 32; ++i) {
        const u32x2 x = read_column(va[i] + (r + 16 * n) * (2 * DP));
        const u32x2 y = read_column(va[i] + (r + 16 * n + 8) * (2 * DP));
        o[i] = Mfma<T>::mul(u32x4{x[0], x[1], y[0], y[1]}, pb, o[i]);
      }
    }
  }
};

// A wavefront's 16 rows, for the 16 x 16 instructions: a row's keys are in four lanes, lane / 16 = 0 .. 3,
// and half as many of them in each as of 32 rows, whose other half would be worked on for nothing.
template <typename T>
struct Mfma16;
template <>
struct Mfma16<_Float16> {
  __device__ static __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma16<__bf16> {
  __device__ static __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
  }
};

__device__ __forceinline__ float max_of_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_of_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

template <typename T, int DP, int DC = DP>
struct Rows16 {
  u32x4 q[DC / 32];                    // operand columns: row lane % 16, elements 32 i + 8 (lane / 16) ..
  f32x4 o[DC / 16];                    // element j of o[i]: row lane % 16, output 16 i + 4 (lane / 16) + j
  float m, l;                          // as in Rows
  u32 ka[DC / 32], va[DC / 16];        // LDS addresses that this lane reads of a tile of 32 keys

  __device__ __forceinline__ void start(const T* qp, int D, u32 flip) {
    const int quarter = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) {
      const int c = 32 * i + 8 * quarter;
      q[i] = *(c < D ? reinterpret_cast<const u32x4*>(qp + c) : reinterpret_cast<const u32x4*>(kZeros)) ^ flip;
    }
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void addresses(u32 lk, u32 lv) {
    const int lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) ka[i] = lk + row * (2 * DP) + 16 * ((4 * i + quarter) ^ place_k<DP>(row));
    const int key = 4 * quarter + (row >> 2);
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) {
      const int c = 2 * i + ((row & 3) >> 1);
      va[i] = lv + key * (2 * DP) + 16 * (c ^ place_v16<DP>(key)) + 8 * (row & 1);
    }
  }
  // Products of 16 keys from row r (0 or 16) of a tile on: element j is key 4 (lane / 16) + j.
  __device__ __forceinline__ f32x4 scores(int r) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < DC / 32; ++i) s = Mfma16<T>::mul(read_lds16(ka[i] + r * (2 * DP)), q[i], s);
    return s;
  }
  // Scores of 32 keys -> probabilities, as the next product's operand; the rest as in Rows.
  template <typename F>
  __device__ __forceinline__ u32x4 softmax(f32x4 (&s)[2], float c, float lift, bool masked, F seen) {
    const int quarter = (threadIdx.x >> 4) & 3;
    if (masked) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = seen(16 * n + 4 * quarter + j) ? s[n][j] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, s[n][j]);
    top = max_of_quarters(top);
    if (__ballot((top - m) * c > 8.0f + kLift<T> || (m == -INFINITY && top > m))) {
      const float m_new = fmaxf(m, kLift<T> == 0 ? top : top - lift);
      // (rows that have seen no key yet keep their zeros)
      const float keep = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - m_new) * c);
      m = m_new;
      l *= keep;
#pragma unroll
      for (int i = 0; i < DC / 16; ++i) o[i] *= keep;
    }
    const float base = m == -INFINITY ? 0.f : -m * c;
    u32x4 p;
    float sum = 0.f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[n][j], c, base));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[n][j + 1], c, base));
        sum += p0 + p1;
        p[2 * n + j / 2] = two_rounded<T>(p0, p1);
      }
    l += sum;
    return p;
  }
  // O^T += V^T P^T for the tile's 32 keys: a lane's 8 of an operand are 4 quarter .. + 3 and 16 behind
  // those, as its probabilities lie.
  __device__ __forceinline__ void values(u32x4 p) {
#pragma unroll
    for (int i = 0; i < DC / 16; ++i) {
      const u32x2 x = read_column(va[i]), y = read_column(va[i] + 16 * (2 * DP));
      o[i] = Mfma16<T>::mul(u32x4{x[0], x[1], y[0], y[1]}, p, o[i]);
    }
  }
};

}  // namespace tdq
