// kv_attn.hpp -- what the kernels of the attention over quantized pages share.
#pragma once

#include "kv.hpp"

namespace mpq {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
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
  float* part_ml;     // [tile][split][16][2]
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

__device__ __forceinline__ float across(float v, int mask) { return __shfl_xor(v, mask, 64); }

#endif

}  // namespace mpq
