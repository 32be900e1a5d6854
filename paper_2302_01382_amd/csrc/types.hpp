// types.hpp -- element types of the serving calls: fp32, bf16 and fp16 in memory, fp32 in registers.
#pragma once

#include "common.hpp"

namespace mpq {

inline bool known_type(int type) { return type == MPQ_F32 || type == MPQ_BF16 || type == MPQ_F16; }
inline int type_size(int type) { return type == MPQ_F32 ? 4 : 2; }

#if defined(__HIPCC__)

typedef int v2i __attribute__((ext_vector_type(2)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
// in memory at any address that an element may have
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef _Float16 f16x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int T>
struct Elem;
template <>
struct Elem<MPQ_F32> {
  typedef float type;
  static __device__ __forceinline__ f32x8 load8(const float* p) {
    const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4_any*>(p); }
  static __device__ __forceinline__ void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4_any*>(p) = v; }
  static __device__ __forceinline__ void store8(float* p, f32x8 v) {
    store4(p, __builtin_shufflevector(v, v, 0, 1, 2, 3));
    store4(p + 4, __builtin_shufflevector(v, v, 4, 5, 6, 7));
  }
};
template <>
struct Elem<MPQ_BF16> {
  typedef __bf16 type;
  static __device__ __forceinline__ f32x8 load8(const __bf16* p) {
    return __builtin_convertvector((bf16x8)*reinterpret_cast<const bf16x8_any*>(p), f32x8);
  }
  static __device__ __forceinline__ f32x4 load4(const __bf16* p) {
    return __builtin_convertvector((bf16x4)*reinterpret_cast<const bf16x4_any*>(p), f32x4);
  }
  static __device__ __forceinline__ void store4(__bf16* p, f32x4 v) {
    *reinterpret_cast<bf16x4_any*>(p) = __builtin_convertvector(v, bf16x4);
  }
  static __device__ __forceinline__ void store8(__bf16* p, f32x8 v) {
    *reinterpret_cast<bf16x8_any*>(p) = __builtin_convertvector(v, bf16x8);
  }
};
template <>
struct Elem<MPQ_F16> {
  typedef _Float16 type;
  static __device__ __forceinline__ f32x8 load8(const _Float16* p) {
    return __builtin_convertvector((f16x8)*reinterpret_cast<const f16x8_any*>(p), f32x8);
  }
  static __device__ __forceinline__ f32x4 load4(const _Float16* p) {
    return __builtin_convertvector((f16x4)*reinterpret_cast<const f16x4_any*>(p), f32x4);
  }
  static __device__ __forceinline__ void store4(_Float16* p, f32x4 v) {
    *reinterpret_cast<f16x4_any*>(p) = __builtin_convertvector(v, f16x4);
  }
  static __device__ __forceinline__ void store8(_Float16* p, f32x8 v) {
    *reinterpret_cast<f16x8_any*>(p) = __builtin_convertvector(v, f16x8);
  }
};

// bit_constants, but a maximum so small that inv would not be finite (below qmax / FLT_MAX, 4e-37) counts as 0
__device__ __forceinline__ void step_constants(float m, int bits, float& scale, float& inv) {
  bit_constants(m, bits, scale, inv);
  if (inv == __builtin_inff()) scale = inv = 0.0f;
}

// the low bytes of t = 1.5 * 2^23 + code, which are the codes
__device__ __forceinline__ unsigned low_bytes(float a, float b, float c, float d) {
  const unsigned lo = __builtin_amdgcn_perm((unsigned)bits_from_f(b), (unsigned)bits_from_f(a), 0x0c0c0400u);
  const unsigned hi = __builtin_amdgcn_perm((unsigned)bits_from_f(d), (unsigned)bits_from_f(c), 0x04000c0cu);
  return lo | hi;
}

// four codes of Eq. 1 as the bytes of a dword, the first in the lowest
__device__ __forceinline__ unsigned pack_codes(float a, float b, float c, float d, float inv, float qmax) {
  return ((unsigned)(int)code_f(a, inv, qmax) & 0xFFu) | (((unsigned)(int)code_f(b, inv, qmax) & 0xFFu) << 8) |
         (((unsigned)(int)code_f(c, inv, qmax) & 0xFFu) << 16) | ((unsigned)(int)code_f(d, inv, qmax) << 24);
}

#endif  // __HIPCC__

}  // namespace mpq
