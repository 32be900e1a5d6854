// kv_attn.hpp -- what the kernels of the attention over quantized pages share.
#pragma once

#include "attn_span.hpp"
#include "kv.hpp"

namespace mpq {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
// of a split's row: maximum, sum, and the exponent of the power of two that its share of the output is in units of
struct Partial {
  float m, l, e;
};
struct AttnArgs {
  mpq_kv_cache c;
  mpq_kv_batch b;
  const void* q;
  int64_t q_ts, q_hs;
  void* out;
  int64_t o_ts, o_hs;
  int q_heads, group, causal;
  int64_t window;
  float scale;        // softmax_scale
  int64_t row_tiles;  // tiles of 16 (row, query head) pairs per sequence and key head
  int splits;
  int tile_rows;      // of a tile that a sequence may have: 16 but where there is a single tile
  float* part_o;      // splits > 1: [tile][split][16][dim], then
  Partial* part;      // [tile][split][16]
};

// defined in kv_prompt.hip: the most rows of a workgroup there, and the launch of wg_tiles row tiles of wg_rows (those, or for
// dim <= 128 also 64) per sequence and key head
int prompt_rows(int type, int dim);
int launch_prompt(int type, const AttnArgs& a, int64_t wg_tiles, int wg_rows, bool prepare_only, hipStream_t st);

#if defined(__HIPCC__)

// four codes -> fp16: the byte code + 128 as the low bits of 1024 + u, less 1152 (both exact)
__device__ __forceinline__ void codes4(int w, f16x2& lo, f16x2& hi) {
  const unsigned u = (unsigned)w ^ 0x80808080u;
  const f16x2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
  lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
  hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
}
__device__ __forceinline__ f16x8 codes8(int a, int b) {
  f16x2 x, y, z, w;
  codes4(a, x, y);
  codes4(b, z, w);
  return f16x8{x.x, x.y, y.x, y.y, z.x, z.y, w.x, w.y};
}

// The digits of g: g % a, g / a % b, g / a / b % c, g / a / b / c.  A division in 64 bits is 150 scalar instructions, which a
// wave has to itself here, so that they are done in 32 where the grid is that small (one token of one sequence of 384 tokens:
// with the rows' divisions 8.9 -> 7.9 us).
struct Digits {
  int64_t d[4];
};
template <typename I>
__device__ __forceinline__ Digits split_digits(I g, I a, I b, I c) {
  Digits r;
  r.d[0] = (int64_t)(g % a);
  g /= a;
  r.d[1] = (int64_t)(g % b);
  g /= b;
  r.d[2] = (int64_t)(g % c);
  r.d[3] = (int64_t)(g / c);
  return r;
}
__device__ __forceinline__ Digits digits(int64_t a, int64_t b, int64_t c) {
  if (gridDim.z == 1) return split_digits<unsigned>(blockIdx.x, (unsigned)a, (unsigned)b, (unsigned)c);
  return split_digits<uint64_t>((uint64_t)block_index(), (uint64_t)a, (uint64_t)b, (uint64_t)c);
}

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((unsigned)a / (unsigned)b) : a / b;
}

__device__ __forceinline__ f32x4 times_two_to(f32x4 v, int e) {
  return f32x4{__builtin_ldexpf(v.x, e), __builtin_ldexpf(v.y, e), __builtin_ldexpf(v.z, e), __builtin_ldexpf(v.w, e)};
}

__device__ __forceinline__ float across(float v, int mask) { return __shfl_xor(v, mask, 64); }

#endif

}  // namespace mpq
