// rotate_heads.hip -- queries and keys on their way from the linear layer to the cache: a norm per head and the rotation by
// position, in one read and one write.
//
// y = x / sqrt(mean x^2 + eps) * w, then pairs (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = position * frequency.  A lane
// holds eight channels of a head that make four whole pairs, so that the rotation needs no other lane, and the norm a sum over the
// lanes of the head; a wave takes 64 / LPH heads of a row at a time.  Cosines and sines depend on the row alone: a lane makes its
// four once per row.  The angle in turns is a product in 64 bits less its nearest whole number: a position of a million times a
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

// LPH: lanes of a head, dim / 8 rounded up to a power of two.  NEIGHBOURS: pairs are channels 2 j and 2 j + 1.
template <int T, int LPH, bool NEIGHBOURS>
__global__ __launch_bounds__(kBlock) void rotate_heads_k(RotateArgs a) {
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int HPW = kWave / LPH;
  const int lane = threadIdx.x & 63, u = lane % LPH;
  const int64_t wave = block_index() * (kBlock / kWave) + (threadIdx.x >> 6);
  const int64_t row = wave / a.per_row;
  if (row >= a.rows) return;  // uniform over the wave
  const bool real = u < a.dim / 8, turns = u < a.pairs / 4;
  // the lane's channels: four from `first` on and four from `second` on
  const int first = NEIGHBOURS || !turns ? 8 * u : 4 * u, second = NEIGHBOURS || !turns ? first + 4 : first + a.pairs;
  float c[4], s[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = 1.0f;
    s[j] = 0.0f;
  }
  if (turns) {
    const double position = (double)a.positions[row] * 0.15915494309189535;  // 1 / (2 pi)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double t = position * (double)a.frequencies[4 * u + j];
      sincospif(2.0f * (float)(t - __builtin_rint(t)), &s[j], &c[j]);
    }
  }
  const int heads = a.heads[0] + a.heads[1];
  const float one_of = 1.0f / (float)a.dim;
  int h = (int)(wave - row * a.per_row) * a.run * HPW + lane / LPH;
  for (int g = 0; g < a.run; ++g, h += HPW) {
    const int which = h < a.heads[0] ? 0 : 1;
    const int64_t head = h - (which ? a.heads[0] : 0);
    const bool mine = real && h < heads;
    f32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
    if (mine) {
      const El* from = reinterpret_cast<const El*>(a.in[which]) + row * a.in_ts[which] + head * a.in_hs[which];
      x = E::load4(from + first);
      y = E::load4(from + second);
    }
    const float* weight = a.weight[which];
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(x[e], x[e], __builtin_fmaf(y[e], y[e], sum));
#pragma unroll
    for (int m = 1; m < LPH; m <<= 1) sum += __shfl_xor(sum, m, 64);
    if (!mine) continue;
    if (weight) {
      const float mean = __builtin_fmaf(sum, one_of, a.eps);
      float r = __builtin_amdgcn_rsqf(mean);  // (to one step; the line below to about half of one)
      r = __builtin_fmaf(0.5f * r, __builtin_fmaf(-mean * r, r, 1.0f), r);
      x = x * r * Elem<MPQ_F32>::load4(weight + first);
      y = y * r * Elem<MPQ_F32>::load4(weight + second);
    }
    if (turns) {
      f32x4 p, q;
      if (NEIGHBOURS) {
        p = f32x4{x[0], x[2], y[0], y[2]};
        q = f32x4{x[1], x[3], y[1], y[3]};
      } else {
        p = x;
        q = y;
      }
      f32x4 v, w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = __builtin_fmaf(p[e], c[e], -(q[e] * s[e]));
        w[e] = __builtin_fmaf(q[e], c[e], p[e] * s[e]);
      }
      if (NEIGHBOURS) {
        x = f32x4{v[0], w[0], v[1], w[1]};
        y = f32x4{v[2], w[2], v[3], w[3]};
      } else {
        x = v;
        y = w;
      }
    }
    El* to = reinterpret_cast<El*>(a.out[which]) + row * a.out_ts[which] + head * a.out_hs[which];
    E::store4(to + first, x);
    E::store4(to + second, y);
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
  const int per_wave = kWave / lanes, groups = (a.heads[0] + a.heads[1] + per_wave - 1) / per_wave;
  a.run = groups;
  while (a.run > 1 && a.rows * ((groups + a.run - 1) / a.run) < 4 * 2 * kNumCU) a.run = (a.run + 1) / 2;
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
    if (a.heads[i] == 0) continue;
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
  if (blocks_z(rows * (((int64_t)q_heads + k_heads + 1) / 2), kBlock) > 65535u) return MPQ_ERR_SHAPE;
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) return launch<MPQ_F32>(a, layout, st);
  if (type == MPQ_BF16) return launch<MPQ_BF16>(a, layout, st);
  return launch<MPQ_F16>(a, layout, st);
}
