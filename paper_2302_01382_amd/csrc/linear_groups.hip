// linear_groups.hip -- a linear layer of few rows whose 4-bit weights have a step per group of 32, 64 or 128 input channels.
//
// y[m][n] = act(sum_g s[n][g] sum_{k in g} c[n][k] x[m][k]).  The weights are read once and meet at most 64 rows, so that their bytes
// bound it.  No LDS tiles: a lane loads 16 bytes, 32 codes, of a weight row; the waves of a workgroup deal out k in steps of 256 (a
// whole cache line of a weight row) and their sums meet in LDS, in a fixed order.
//
// The product runs on v_mfma_f32_16x16x32 in the rows' own 16-bit type (rows x times codes): bf16 and fp16 hold x and codes exactly.
// fp32 rows go in as three bf16 terms, 24 bits.  Both types take a code's four bits as they are: u = code + 8 in the mantissa of 16,
// which makes 16 + u = code + 24, one shift and one three-operand logic instruction for two codes.  The 24 comes off again in the same sums: they
// start from -24 times the sum of the group's x, a matrix step with a constant operand that all channels share.  A sum's rounding is that
// of terms up to 24 / 4 times as large as without it, 2^-21 of them.
//
// A group's sum has to hold that group alone, and a matrix step adds up the k of four quarters of the wave.  A lane's 16 bytes are
// 32 neighbouring codes: for groups of 128, whose four quarters are one group, operand c is dword c of every lane and x is read to
// match; for 64 and 32 the quarters exchange their dwords, four swaps for four dwords, after which step c has 32 neighbouring k.
#include "qgemm_dma.hpp"

namespace mpq {

struct GroupsArgs {
  const void* x;
  int64_t x_stride;
  const uint8_t* w;
  const void* scale;
  int64_t M, N;
  int K, act, y_type;
  void* y;
};

constexpr int kGroupWaves = 8, kGroupThreads = kGroupWaves * 64, kGroupStep = 256;

template <int T>
struct Operand {  // bf16, also for the terms of fp32
  static constexpr int TERMS = T == MPQ_F32 ? 3 : 1, SHIFT = 3;
  static constexpr unsigned MASK = 0x00780078u, FORM = 0x41804180u ^ 0x00400040u;  // 16, and the codes' sign bits turned: u = code + 8
  static constexpr unsigned MINUS = 0xC1C0C1C0u;                                   // -24
  static __device__ __forceinline__ f32x4 mfma(v4i a, v4i b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Operand<MPQ_F16> {
  static constexpr int TERMS = 1, SHIFT = 6;
  static constexpr unsigned MASK = 0x03C003C0u, FORM = 0x4C004C00u ^ 0x02000200u, MINUS = 0xCE00CE00u;
  static __device__ __forceinline__ f32x4 mfma(v4i a, v4i b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// Eight codes as an operand: its dword i holds codes i and i + 4.
template <int T>
__device__ __forceinline__ v4i codes_operand(unsigned w) {
  using O = Operand<T>;
  v4i r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = O::SHIFT - 4 * i;
    const unsigned v = left >= 0 ? w << (left & 31) : w >> (-left & 31);
    r[i] = (int)((v & O::MASK) ^ O::FORM);
  }
  return r;
}
// eight 16-bit values in their order -> the order of codes_operand
__device__ __forceinline__ v4i pair_up(v4i v) {
  return v4i{(int)__builtin_amdgcn_perm((unsigned)v.z, (unsigned)v.x, 0x05040100u), (int)__builtin_amdgcn_perm((unsigned)v.z, (unsigned)v.x, 0x07060302u),
             (int)__builtin_amdgcn_perm((unsigned)v.w, (unsigned)v.y, 0x05040100u), (int)__builtin_amdgcn_perm((unsigned)v.w, (unsigned)v.y, 0x07060302u)};
}

// Dword d of quarter c becomes dword c of quarter d.
__device__ __forceinline__ v4i exchange(v4i v) {
  const auto a = __builtin_amdgcn_permlane32_swap((unsigned)v.x, (unsigned)v.z, false, false);
  const auto b = __builtin_amdgcn_permlane32_swap((unsigned)v.y, (unsigned)v.w, false, false);
  const auto c = __builtin_amdgcn_permlane16_swap((unsigned)a[0], (unsigned)b[0], false, false);
  const auto d = __builtin_amdgcn_permlane16_swap((unsigned)a[1], (unsigned)b[1], false, false);
  return v4i{(int)c[0], (int)c[1], (int)d[0], (int)d[1]};
}

template <int S>
__device__ __forceinline__ float step_at(const void* p, int64_t i) {
  return (float)reinterpret_cast<const typename Elem<S>::type*>(p)[i];
}

// T: type of x, S: of the steps, G: group.  A workgroup takes NT x 16 output channels and MT x 16 rows.
// grid: x channels, y blocks of rows
template <int T, int S, int G, int MT, int NT>
__global__ __launch_bounds__(kGroupThreads, 2) void linear_groups_k(GroupsArgs p) {
  using O = Operand<T>;
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int NW = kGroupWaves, TERMS = O::TERMS;
  __shared__ f32x4 red[NW][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT), m0 = (int64_t)blockIdx.y * (16 * MT);
  const int K = p.K, groups = K / G;
  const int rows = (int)(p.M - m0 < 16 * MT ? p.M - m0 : 16 * MT);
  // channels and rows past the edge re-read the last one; never stored
  const uint8_t* w_row[NT];
  int64_t s_row[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t n = n0 + j * 16 + r < p.N ? n0 + j * 16 + r : p.N - 1;
    w_row[j] = p.w + n * (K >> 1);
    s_row[j] = n * groups;
  }
  const El* x_row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = i * 16 + r;
    x_row[i] = reinterpret_cast<const El*>(p.x) + (m0 + (m < rows ? m : rows - 1)) * p.x_stride;
  }
  f32x4 total[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) total[i][j] = f32x4{0, 0, 0, 0};

  const int steps = (K + kGroupStep - 1) / kGroupStep;
  constexpr int PER = G / 32;  // matrix steps of a group
  const v4i minus = {(int)O::MINUS, (int)O::MINUS, (int)O::MINUS, (int)O::MINUS};
  for (int s = wave; s < steps; s += NW) {
    v4i w[NT][2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      // a lane's 32 codes lie in the row or behind it, as a whole; those behind are not multiplied
      const int k = s * kGroupStep + 128 * half + 32 * q, at = k < K ? k : K - 32;
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j][half] = *reinterpret_cast<const v4i_byte*>(w_row[j] + (at >> 1));
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int k1 = s * kGroupStep + 128 * half;
      if (G < 128) {
#pragma unroll
        for (int j = 0; j < NT; ++j) w[j][half] = exchange(w[j][half]);
      }
#pragma unroll
      for (int c0 = 0; c0 < 4; c0 += PER) {
        const int g = (k1 + 32 * c0) / G;
        if (g >= groups) break;  // uniform
        v4i x[PER][MT][TERMS];
        f32x4 from[MT];  // -24 times the sum of the group's x
#pragma unroll
        for (int i = 0; i < MT; ++i) from[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < PER; ++c) {
          const El* chunk[MT];
#pragma unroll
          for (int i = 0; i < MT; ++i) chunk[i] = x_row[i] + k1 + (G < 128 ? 32 * (c0 + c) + 8 * q : 32 * q + 8 * c);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            if constexpr (T == MPQ_F32) {
              f32x8 v = E::load8(chunk[i]);
#pragma unroll
              for (int t = 0; t < TERMS; ++t) {
                const bf16x8 top = __builtin_convertvector(v, bf16x8);
                x[c][i][t] = pair_up(__builtin_bit_cast(v4i, top));
                v -= __builtin_convertvector(top, f32x8);
              }
            } else {
              x[c][i][0] = pair_up(*reinterpret_cast<const v4i_byte*>(chunk[i]));
            }
#pragma unroll
            for (int t = 0; t < TERMS; ++t) from[i] = O::mfma(x[c][i][t], minus, from[i]);
          }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          f32x4 part[MT];
#pragma unroll
          for (int i = 0; i < MT; ++i) part[i] = from[i];
#pragma unroll
          for (int c = 0; c < PER; ++c) {
            const v4i codes = codes_operand<T>((unsigned)w[j][half][c0 + c]);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
              for (int t = 0; t < TERMS; ++t) part[i] = O::mfma(x[c][i][t], codes, part[i]);
          }
          const float sw = step_at<S>(p.scale, s_row[j] + g);
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) total[i][j][e] = __builtin_fmaf(part[i][e], sw, total[i][j][e]);
        }
      }
    }
  }
  // the waves' sums, a row tile at a time: lane (channel r, rows 4 q .. 4 q + 3)
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    if (i) __syncthreads();
#pragma unroll
    for (int j = 0; j < NT; ++j) red[wave][j][lane] = total[i][j];
    __syncthreads();
    for (int t = threadIdx.x; t < NT * 64; t += kGroupThreads) {
      const int j = t >> 6, l = t & 63;
      f32x4 sum = red[0][j][l];
#pragma unroll
      for (int v = 1; v < NW; ++v) sum += red[v][j][l];
      const int64_t n = n0 + j * 16 + (l & 15);
      if (n >= p.N) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = i * 16 + 4 * (l >> 4) + e;
        if (m >= rows) continue;
        const float y = apply_act(sum[e], p.act);
        const int64_t to = (m0 + m) * p.N + n;
        if (p.y_type == MPQ_F32) reinterpret_cast<float*>(p.y)[to] = y;
        else reinterpret_cast<unsigned short*>(p.y)[to] = to_half(y, p.y_type == MPQ_BF16);
      }
    }
  }
}

template <int T, int S, int G>
static int go(const GroupsArgs& p, hipStream_t st) {
  const int64_t row_tiles = (p.M + 15) / 16;
  const dim3 grid((unsigned)((p.N + 15) / 16), (unsigned)((p.M + 63) / 64));
  if (row_tiles == 1) linear_groups_k<T, S, G, 1, 1><<<grid, kGroupThreads, 0, st>>>(p);
  else if (row_tiles == 2) linear_groups_k<T, S, G, 2, 1><<<grid, kGroupThreads, 0, st>>>(p);
  else linear_groups_k<T, S, G, 4, 1><<<grid, kGroupThreads, 0, st>>>(p);
  return launch_status();
}
template <int T, int S>
static int go_group(const GroupsArgs& p, int group, hipStream_t st) {
  return group == 32 ? go<T, S, 32>(p, st) : group == 64 ? go<T, S, 64>(p, st) : go<T, S, 128>(p, st);
}
template <int T>
static int go_type(const GroupsArgs& p, int group, int scale_type, hipStream_t st) {
  if (scale_type == MPQ_F32) return go_group<T, MPQ_F32>(p, group, st);
  return scale_type == MPQ_BF16 ? go_group<T, MPQ_BF16>(p, group, st) : go_group<T, MPQ_F16>(p, group, st);
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_linear_groups(const void* x, int x_type, int64_t M, int64_t N, int64_t K, int64_t x_stride, const uint8_t* w_q,
                                 int group, const void* w_scale, int scale_type, int act, int y_type, void* y_out, void* stream) {
  if (!known_type(x_type) || !known_type(scale_type) || !known_type(y_type) || act < MPQ_ACT_NONE || act > MPQ_ACT_GELU) return MPQ_ERR_SHAPE;
  if (group != 32 && group != 64 && group != 128) return MPQ_ERR_SHAPE;
  if (M < 0 || N <= 0 || K <= 0 || K % group || K > (1 << 30) || x_stride < K) return MPQ_ERR_SHAPE;
  if (mul_overflows(M, x_stride) || mul_overflows(N, K) || mul_overflows(M, N)) return MPQ_ERR_SHAPE;
  // (a grid counts 2^32 threads in x and 65535 blocks of rows in y)
  if (N > (1 << 26) || (M + 63) / 64 > kMaxGridY) return MPQ_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(x) & (uintptr_t)(type_size(x_type) - 1)) return MPQ_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(w_scale) & (uintptr_t)(type_size(scale_type) - 1)) return MPQ_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(y_out) & (uintptr_t)(type_size(y_type) - 1)) return MPQ_ERR_ALIGN;
  if (M == 0) return MPQ_OK;
  if (!x || !w_q || !w_scale || !y_out) return MPQ_ERR_NULL;
  const GroupsArgs p{x, x_stride, w_q, w_scale, M, N, (int)K, act, y_type, y_out};
  hipStream_t st = (hipStream_t)stream;
  if (x_type == MPQ_F32) return go_type<MPQ_F32>(p, group, scale_type, st);
  return x_type == MPQ_BF16 ? go_type<MPQ_BF16>(p, group, scale_type, st) : go_type<MPQ_F16>(p, group, scale_type, st);
}
