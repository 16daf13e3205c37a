// Element types of the 8-bit linear, the head norm and the attention: binary16, bfloat16 and
// binary32 read as floats, floats rounded to them, and direct-to-LDS copies.
#pragma once

#include "tdq_internal.hpp"

namespace tdq {

typedef unsigned int u32;
typedef unsigned short u16;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
// (aligned to an element only: the memory path takes such loads and stores in one instruction)
typedef u32 u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef u32 u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// Grid of n workgroups: an axis holds fewer than 2^32 threads (workgroups past the last return).
inline dim3 two_axes(long long n) {
  const long long axis = 1 << 22;
  return dim3(n < axis ? (unsigned)n : (unsigned)axis, (unsigned)((n + axis - 1) / axis));
}

// Two adjacent 16-bit elements as floats, and back (to nearest, ties to even).
template <typename T>
__device__ __forceinline__ f32x2 two_floats(u32 w);
template <>
__device__ __forceinline__ f32x2 two_floats<_Float16>(u32 w) {
  const h16x2 h = __builtin_bit_cast(h16x2, w);
  return f32x2{(float)h[0], (float)h[1]};
}
template <>
__device__ __forceinline__ f32x2 two_floats<__bf16>(u32 w) {
  return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
}
template <typename T>
__device__ __forceinline__ u32 two_rounded(float a, float b);
template <>
__device__ __forceinline__ u32 two_rounded<_Float16>(float a, float b) {
  return __builtin_bit_cast(u32, h16x2{(_Float16)a, (_Float16)b});
}
template <>
__device__ __forceinline__ u32 two_rounded<__bf16>(float a, float b) {
  return __builtin_bit_cast(u32, b16x2{(__bf16)a, (__bf16)b});
}

// V consecutive elements (4 or 8) from an address aligned to an element, as floats; and back.
template <typename T, int V>
__device__ __forceinline__ void load_floats(const T* p, float (&x)[V]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const u32x4_any w = *reinterpret_cast<const u32x4_any*>(p + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i + j] = __uint_as_float(w[j]);
    }
  } else {
    u32 w[V / 2];
    if constexpr (V == 8) {
      const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = v[j];
    } else {
      const u32x2_any v = *reinterpret_cast<const u32x2_any*>(p);
      w[0] = v[0];
      w[1] = v[1];
    }
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const f32x2 f = two_floats<T>(w[j]);
      x[2 * j] = f[0];
      x[2 * j + 1] = f[1];
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_floats(T* p, const float (&x)[V]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      u32x4_any w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(x[i + j]);
      *reinterpret_cast<u32x4_any*>(p + i) = w;
    }
  } else if constexpr (V == 8) {
    u32x4_any w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = two_rounded<T>(x[2 * j], x[2 * j + 1]);
    *reinterpret_cast<u32x4_any*>(p) = w;
  } else {
    u32x2_any w;
    w[0] = two_rounded<T>(x[0], x[1]);
    w[1] = two_rounded<T>(x[2], x[3]);
    *reinterpret_cast<u32x2_any*>(p) = w;
  }
}

// 64 pieces of 16 bytes, one address a lane, to 1024 consecutive bytes of LDS from lds_base on
// (the same in every lane).  The compiler neither sees that this writes LDS nor counts it: the
// kernel waits for it (vmcnt) and orders it against the LDS accesses of others (barrier) itself.
__device__ __forceinline__ void copy_to_lds(const void* p, u32 lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(p), "s"(lds_base)
               : "memory");
}
// The same with a base that is the same in every lane and 32-bit byte offsets.
__device__ __forceinline__ void copy_to_lds(const void* base, u32 off, u32 lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds_base)
               : "memory");
}
// The same for what is read once: it takes no place in the caches from what others read again.
__device__ __forceinline__ void stream_to_lds(const void* base, u32 off, u32 lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
               :
               : "v"(off), "s"(base), "s"(lds_base)
               : "memory");
}
// 64 floats, one offset a lane, to 256 consecutive bytes of LDS.
__device__ __forceinline__ void copy_float_to_lds(const void* base, u32 off, u32 lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds_base)
               : "memory");
}
// Everything copied by this wavefront has arrived.
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ u32 lds_address(const void* p) {
  return (u32)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

}  // namespace tdq
