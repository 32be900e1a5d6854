// rotate_heads.hip -- queries and keys on their way from the linear layer to the cache: a norm per head and the rotation by
// position, in one read and one write.
//
// y = x / sqrt(mean x^2 + eps) * w, then pairs (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = position * frequency.  A lane
// holds eight channels of a head that make four whole pairs, so that the rotation needs no other lane, and the norm a sum over the
// lanes of the head; a wave takes 64 / LPH heads of a row at a time.  Cosines and sines depend on the row alone: a wave makes each
// once, a pair to a lane, and hands them round.  Bytes bound it (12289 x 40 x 128 fp16: 252 MB in 55 us, 4.6 TB/s; a large copy reaches
// 5.2), and with few rows the host.  The angle in turns is a product in 64 bits less its nearest whole number: a position of a million times a
// frequency of one is 2e5 turns, of which fp32 would keep seven bits.
#include "types.hpp"

namespace mpq {

struct RotateArgs {
  const void* in[2];  // q, k
  void* out[2];
  int64_t in_ts[2], in_hs[2], out_ts[2], out_hs[2];
  const float* weight[2];
  int heads[2];
  const int32_t* positions;
  const float* frequencies;
  int64_t rows;
  int dim, pairs, per_row, run;  // waves to a row, groups of heads to a wave
  float eps;
};

// sum over each aligned group of LPH lanes
template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
  v += dpp<kQuadSwap1>(v);
  if (LPH >= 4) v += dpp<kQuadSwap2>(v);
  if (LPH >= 8) v += dpp<kRowHalfMirror>(v);
  if (LPH >= 16) v += dpp<kRowMirror>(v);
  if (LPH == 32) v += __shfl_xor(v, 16, 64);
  return v;
}

__device__ __forceinline__ int64_t uniform(int64_t v) {
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)v), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// LPH: lanes of a head, dim / 8 rounded up to a power of two.  NEIGHBOURS: pairs are channels 2 j and 2 j + 1.
template <int T, int LPH, bool NEIGHBOURS>
__global__ __launch_bounds__(kBlock) void rotate_heads_k(RotateArgs a) {
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int HPW = kWave / LPH;
  const int lane = threadIdx.x & 63, u = lane % LPH;
  const int64_t wave = block_index() * (kBlock / kWave) + (threadIdx.x >> 6);
  const int64_t row = uniform(wave / a.per_row);
  if (row >= a.rows) return;  // uniform over the wave
  const bool real = u < a.dim / 8, turns = u < a.pairs / 4;
  // the lane's channels: four from `first` on and four from `second` on
  const bool together = NEIGHBOURS || !turns;
  const int first = together ? 8 * u : 4 * u, second = together ? first + 4 : first + a.pairs;
  // groups of HPW heads, q's before k's: which a group is of, and where it lies, is the same for the whole wave
  const int of_q = (a.heads[0] + HPW - 1) / HPW, groups = of_q + (a.heads[1] + HPW - 1) / HPW;
  const int g0 = __builtin_amdgcn_readfirstlane((int)(wave - row * a.per_row)) * a.run, g1 = g0 + a.run < groups ? g0 + a.run : groups;
  const int sub = lane / LPH;
  auto load = [&](int g) {
    const int which = g < of_q ? 0 : 1, head = (which ? g - of_q : g) * HPW;
    f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (real && head + sub < a.heads[which]) {
      const El* from = reinterpret_cast<const El*>(a.in[which]) + row * a.in_ts[which] + head * a.in_hs[which] + sub * a.in_hs[which];
      if (NEIGHBOURS) v = E::load8(from + first);
      else v = __builtin_shufflevector(E::load4(from + first), E::load4(from + second), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return v;
  };
  f32x8 next = {0, 0, 0, 0, 0, 0, 0, 0};
  if (g0 < g1) next = load(g0);
  f32x8 weight[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (a.weight[i] && real)
      weight[i] = __builtin_shufflevector(Elem<MPQ_F32>::load4(a.weight[i] + first), Elem<MPQ_F32>::load4(a.weight[i] + second), 0, 1, 2, 3, 4, 5, 6, 7);
  // a cosine and a sine of every pair, made by one lane each (two where there are more than 64), and handed to the lanes that turn the pair
  float c[4], s[4];
  if (a.pairs > 0) {
    constexpr int EACH = LPH > 16 ? 2 : 1;
    const double position = (double)a.positions[row] * 0.15915494309189535;  // 1 / (2 pi)
    float cs[EACH], sn[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int j = lane + 64 * i;
      const double t = j < a.pairs ? position * (double)a.frequencies[j] : 0.0;
      sincospif(2.0f * (float)(t - __builtin_rint(t)), &sn[i], &cs[i]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int from = 4 * u + j;
      c[j] = __shfl(cs[0], from & 63, 64);
      s[j] = __shfl(sn[0], from & 63, 64);
      if (EACH == 2) {
        const float c1 = __shfl(cs[EACH - 1], from & 63, 64), s1 = __shfl(sn[EACH - 1], from & 63, 64);
        c[j] = from < 64 ? c[j] : c1;
        s[j] = from < 64 ? s[j] : s1;
      }
    }
  }
  const float one_of = 1.0f / (float)a.dim;
  for (int g = g0; g < g1; ++g) {
    const int which = g < of_q ? 0 : 1, head = (which ? g - of_q : g) * HPW;
    f32x8 x = next;
    if (g + 1 < g1) next = load(g + 1);
    if (a.weight[which]) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
      const float mean = __builtin_fmaf(head_sum<LPH>(sum), one_of, a.eps);
      float r = __builtin_amdgcn_rsqf(mean);  // (to one step; the line below to about half of one)
      r = __builtin_fmaf(0.5f * r, __builtin_fmaf(-mean * r, r, 1.0f), r);
      x = x * r * (which ? weight[1] : weight[0]);
    }
    if (turns) {
      constexpr int STEP = NEIGHBOURS ? 2 : 1, OTHER = NEIGHBOURS ? 1 : 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = x[STEP * j], q = x[STEP * j + OTHER];
        x[STEP * j] = __builtin_fmaf(p, c[j], -(q * s[j]));
        x[STEP * j + OTHER] = __builtin_fmaf(q, c[j], p * s[j]);
      }
    }
    if (!real || head + sub >= a.heads[which]) continue;
    El* to = reinterpret_cast<El*>(a.out[which]) + row * a.out_ts[which] + head * a.out_hs[which] + sub * a.out_hs[which];
    if (NEIGHBOURS) {
      E::store8(to + first, x);
    } else {
      E::store4(to + first, __builtin_shufflevector(x, x, 0, 1, 2, 3));
      E::store4(to + second, __builtin_shufflevector(x, x, 4, 5, 6, 7));
    }
  }
}

template <int T, int LPH>
static void go(const RotateArgs& a, int layout, dim3 grid, hipStream_t st) {
  if (layout == MPQ_ROTATE_PAIRS) rotate_heads_k<T, LPH, true><<<grid, kBlock, 0, st>>>(a);
  else rotate_heads_k<T, LPH, false><<<grid, kBlock, 0, st>>>(a);
}

template <int T>
static int launch(RotateArgs& a, int layout, hipStream_t st) {
  const int units = a.dim / 8;
  int lanes = 2;
  while (lanes < units) lanes *= 2;
  const int per_wave = kWave / lanes, groups = (a.heads[0] + per_wave - 1) / per_wave + (a.heads[1] + per_wave - 1) / per_wave;
  // Groups to a wave: all of a row's, which share its angles, halved while there are not four waves to a SIMD (us, two | four | eight | sixteen
  // to a SIMD: 997 x 40 x 128 bf16 8.5 | 8.0 | 8.8 | 8.8, 4000 x 24 x 64 fp32 13.2 | 12.4 | 13.4 | 13.4, 12289 x 40 x 128 fp16 55 | 56 | 56 | 54).
  a.run = groups;
  while (a.run > 1 && a.rows * ((groups + a.run - 1) / a.run) < 16 * kNumCU) a.run = (a.run + 1) / 2;
  a.per_row = (groups + a.run - 1) / a.run;
  const dim3 grid = wide_grid((a.rows * a.per_row + 3) / 4, kBlock);
  switch (lanes) {
    case 2: go<T, 2>(a, layout, grid, st); break;
    case 4: go<T, 4>(a, layout, grid, st); break;
    case 8: go<T, 8>(a, layout, grid, st); break;
    case 16: go<T, 16>(a, layout, grid, st); break;
    default: go<T, 32>(a, layout, grid, st);
  }
  return launch_status();
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_rotate_heads(int type, int64_t rows, int dim, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                                int q_heads, const void* k, int64_t k_token_stride, int64_t k_head_stride, int k_heads,
                                const int32_t* positions, const float* frequencies, int pairs, int layout, const float* q_weight,
                                const float* k_weight, float eps, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                                void* k_out, int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
  if (!known_type(type) || rows < 0 || dim <= 0 || dim > 256 || dim % 16 || q_heads < 0 || k_heads < 0) return MPQ_ERR_SHAPE;
  if (pairs < 0 || pairs % 4 || pairs > dim / 2 || (layout != MPQ_ROTATE_HALVES && layout != MPQ_ROTATE_PAIRS)) return MPQ_ERR_SHAPE;
  if (!(eps >= __FLT_MIN__) || __builtin_isinf(eps)) return MPQ_ERR_SHAPE;
  if ((int64_t)q_heads + k_heads > (1 << 24)) return MPQ_ERR_SHAPE;
  RotateArgs a{{q, k}, {q_out, k_out}, {q_token_stride, k_token_stride}, {q_head_stride, k_head_stride},
               {q_out_token_stride, k_out_token_stride}, {q_out_head_stride, k_out_head_stride}, {q_weight, k_weight}, {q_heads, k_heads},
               positions, frequencies, rows, dim, pairs, 0, 0, eps};
  for (int i = 0; i < 2; ++i) {
    if (a.heads[i] == 0) {  // nothing of it is looked at
      a.weight[i] = nullptr;
      continue;
    }
    if (a.in_ts[i] < 0 || a.in_hs[i] < 0 || a.out_ts[i] < 0 || a.out_hs[i] < 0) return MPQ_ERR_SHAPE;
    if (mul_overflows(rows, a.in_ts[i]) || mul_overflows(rows, a.out_ts[i]) || mul_overflows(a.heads[i], a.in_hs[i]) ||
        mul_overflows(a.heads[i], a.out_hs[i]))
      return MPQ_ERR_SHAPE;
    if (rows > 0 && pieces_overlap(rows, a.out_ts[i], a.heads[i], a.out_hs[i], dim)) return MPQ_ERR_SHAPE;
    if (a.in[i] && a.in[i] == a.out[i] && ((rows > 1 && a.in_ts[i] != a.out_ts[i]) || (a.heads[i] > 1 && a.in_hs[i] != a.out_hs[i])))
      return MPQ_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(a.in[i]) | reinterpret_cast<uintptr_t>(a.out[i])) & (uintptr_t)(type_size(type) - 1)) return MPQ_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(a.weight[i]) & 3u) return MPQ_ERR_ALIGN;
  }
  if ((reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(frequencies)) & 3u) return MPQ_ERR_ALIGN;
  if (mul_overflows(rows, (int64_t)q_heads + k_heads)) return MPQ_ERR_SHAPE;
  if (rows == 0 || q_heads + k_heads == 0) return MPQ_OK;
  if (pairs > 0 && (!positions || !frequencies)) return MPQ_ERR_NULL;
  for (int i = 0; i < 2; ++i)
    if (a.heads[i] > 0 && (!a.in[i] || !a.out[i])) return MPQ_ERR_NULL;
  // an output in the other's place, or in an input's but its own: waves would write the same elements, or read what others have written
  const Pieces in[2] = {{q, q_token_stride, q_heads, q_head_stride}, {k, k_token_stride, k_heads, k_head_stride}};
  const Pieces out[2] = {{q_out, q_out_token_stride, q_heads, q_out_head_stride}, {k_out, k_out_token_stride, k_heads, k_out_head_stride}};
  const int el = (int)type_size(type);
  if (pieces_meet(out[0], out[1], rows, dim, el)) return MPQ_ERR_SHAPE;
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      if (!(i == j && in[i].at == out[i].at) && pieces_meet(out[i], in[j], rows, dim, el)) return MPQ_ERR_SHAPE;
  if (blocks_z(rows * ((int64_t)q_heads + k_heads), kBlock) > 65535u) return MPQ_ERR_SHAPE;
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) return launch<MPQ_F32>(a, layout, st);
  if (type == MPQ_BF16) return launch<MPQ_BF16>(a, layout, st);
  return launch<MPQ_F16>(a, layout, st);
}
